/*
 * vidkv.h - C ABI of the MI355X (gfx950) VidKV hot path:
 *   sub-2-bit KV-cache codec + single-query GQA decode attention over the
 *   packed cache; beside it rotary positions on several axes, a cache in
 *   8 bits with its attention, and trees of drafted tokens checked against it
 *   (second half of this file).
 *
 * Method (arXiv 2503.16257): keys are quantized per channel with mixed
 * precision - the n_anom channels of largest range get the 2-bit uniform
 * group quantizer (Eq. 4), the rest get the FFT-based 1-bit quantizer (Eq. 5;
 * Alg. 3); values get the per-channel ternary quantizer (Eq. 6; Alg. 2) with
 * the most salient visual tokens (Sec. 3.3 (2)) preserved, here in fp16; one
 * decode step computes Softmax(q K^T / sqrt(D)) V over the dequantized cache
 * followed by the fp16 residual tokens (Eq. 3; Alg. 1, Decoding).
 *
 * General rules
 *  - Every pointer named *_dev is DEVICE memory on the current HIP device;
 *    `params` is HOST memory.  The caller owns every buffer; the library
 *    allocates no memory, keeps no pointer after a call returns and never
 *    synchronizes: all work is enqueued on `hip_stream` (a hipStream_t passed
 *    as void*, NULL = the default stream), which must belong to the current
 *    device (else VIDKV_EINVAL).  The library creates no stream and no event
 *    and keeps no state between calls (the one exception is the device array
 *    of vidkv_decode_attention_noalloc).  vidkv_quantize_kv can run part of a
 *    large call beside the rest on a
 *    second stream that the caller hands in (vidkv_side_stream below); without
 *    one, everything runs in line on `hip_stream`.
 *  - All arguments are checked on the host before anything is launched; a
 *    failed check returns a status and launches nothing.  A launch failure
 *    returns VIDKV_EHIP.  Nothing aborts or throws across this boundary.
 *  - Tensors are dense, row-major, fp16 (IEEE binary16) unless stated.
 *    Inputs must be finite; non-finite inputs give unspecified codes and
 *    results (an infinite element of a residual or protected value row, for
 *    one, gives NaN, not infinity, in its channel).  All
 *    stored scales are fp16: a 32-token group of keys whose mean spectral
 *    magnitude (Eq. 5) exceeds 65504 - values of order 10^4 with a common
 *    sign - overflows its scale, with unspecified results for that group.
 *  - Shapes: L = n_layers, B = batch, Hkv = n_kv_heads, Hq = n_q_heads
 *    (Hq % Hkv == 0, Hq / Hkv <= 8; query head h reads KV head h / (Hq/Hkv)),
 *    D = head_dim = 128, G = group = 32, Tq = t_quant (multiple of 32).
 *    One quantize call covers at most 65535 (layer, sequence, KV head)
 *    triples, one decode or flush call at most 65535 sequences (and
 *    sequences x KV heads for a flush); larger shapes return VIDKV_ESHAPE
 *    and are to be split by the caller, e.g. one set of packed buffers (and
 *    one params with n_layers = 1) per layer.
 *  - The byte sizes of the packed buffers come from the vidkv_packed_*_bytes
 *    functions; their layout - every section, record, bit and byte order - is
 *    written down in LAYOUT.md beside this header, and is part of the ABI
 *    version.  Packed buffers and workspaces must
 *    be 256-byte aligned; fp16 tensors and the saliency scores 16-byte
 *    aligned; int32 arrays 4-byte aligned (else VIDKV_EINVAL).
 *  - A workspace is scratch: undefined contents on entry and exit, not to be
 *    shared by calls that may run at the same time.
 */
#ifndef VIDKV_H
#define VIDKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define VIDKV_ABI_VERSION 3

typedef enum {
  VIDKV_OK = 0,
  VIDKV_EINVAL = 1,   /* NULL pointer, bad enum, inconsistent arguments        */
  VIDKV_ESHAPE = 2,   /* a dimension this build does not support               */
  VIDKV_ENOSPACE = 3, /* an output or workspace buffer is too small            */
  VIDKV_EHIP = 4      /* the HIP runtime reported an error at launch           */
} vidkv_status;

/* Hyper-parameters of Alg. 1-3 (G, k, p, gamma) and the cache geometry.
 * Plain data, passed by pointer from host memory, never retained. */
typedef struct vidkv_params {
  int32_t n_layers;      /* L  >= 1                                             */
  int32_t batch;         /* B  >= 1                                             */
  int32_t n_kv_heads;    /* Hkv >= 1                                            */
  int32_t n_q_heads;     /* Hq, multiple of Hkv, Hq/Hkv <= 8                    */
  int32_t head_dim;      /* must be 128                                         */
  int32_t group;         /* G, must be 32 (Sec. 4.1)                            */
  int32_t t_quant;       /* Tq >= 0, multiple of 32: tokens held in packed form */
  int32_t n_anom;        /* 2-bit key channels per head: 0..128, multiple of 8
                            (k * D of Sec. 3.2 (1))                             */
  int32_t use_fft;       /* normal key channels: 1 = FFT-based 1-bit quantizer
                            (Eq. 5), 0 = Eq. 4 at 1 bit on the tokens themselves
                            (the paper's "standard" 1-bit, Sec. 4.1)            */
  int32_t n_salient;     /* protected value tokens per sequence, 0..Tq
                            (n = p * l_v of Sec. 3.3 (2))                       */
  float gamma;           /* ternary threshold factor of Eq. 6 (paper: 0.7)      */
  float softmax_scale;   /* multiplies q.k before the softmax (1/sqrt(128))     */
  int32_t t_capacity;    /* 0: same as t_quant.  Otherwise >= t_quant, multiple
                            of 32: the packed buffers are laid out (and sized)
                            for this many tokens so that vidkv_flush_residual
                            can append blocks in place; every call on the same
                            buffers must pass the same t_capacity              */
  int32_t salient_bits;  /* how the protected value tokens are kept.  0 or 16:
                            verbatim fp16 rows.  2: Alg. 2's STPQuant - the
                            protected rows of a head, gathered in token order,
                            are coded with Eq. 4 at 2 bits per channel over
                            groups of 32 protected tokens (the last group may
                            be shorter)                                        */
  int32_t channel_metric; /* how Alg. 3 ranks the key channels (Sec. 3.2 (1)):
                            0 Range max - min (what the paper adopts), 1
                            Variance, 2 number of Outliers |x| > 3 mean|x|;
                            1 and 2 are the paper's ablation, in float64       */
} vidkv_params;

/* A second stream for the calls that can use one, with the two events that
 * fork it from and join it back into `hip_stream`.  All three are created and
 * owned by the caller, on the device of `hip_stream`, at the default stream
 * priority; the events may have timing disabled.  The call records fork_event
 * on `hip_stream`, lets the side stream wait for it, enqueues part of its work
 * there, records join_event on the side stream and lets `hip_stream` wait for
 * it before anything that depends on that work: to the caller everything
 * stays ordered on `hip_stream`, also under stream capture (the side stream
 * joins the capture and leaves it again within the call).  Once the fork has
 * been recorded the join is enqueued even if a later launch fails.  One such
 * triple serves any number of calls that are enqueued one after another;
 * calls that may be enqueued at the same time from different host threads need
 * one each.  Passing NULL (or using an entry point without the argument)
 * keeps all work in line on `hip_stream`. */
typedef struct vidkv_side_stream {
  void *hip_stream; /* hipStream_t, not the stream the call is enqueued on */
  void *fork_event; /* hipEvent_t */
  void *join_event; /* hipEvent_t */
} vidkv_side_stream;

/* Size queries: pure host functions, usable without a GPU.  Return 0 when
 * `params` is NULL or invalid.  `which`: 0 = quantize_keys, 1 = quantize_values,
 * 2 = decode_attention, 3 = quantize_kv. */
size_t vidkv_packed_keys_bytes(const vidkv_params *params);
size_t vidkv_packed_values_bytes(const vidkv_params *params);
size_t vidkv_workspace_bytes(const vidkv_params *params, int which);

/* Alg. 3 (MixQuant): per (layer, sequence, KV head) rank the 128 channels by
 * range max-min over all Tq tokens (ties: lower channel first), code the top
 * n_anom channels with Eq. 4 at 2 bits (z = min, s = (max-min)/3 per channel
 * and 32-token group, round-half-even) and the others with Eq. 5: a 32-point
 * DFT along the tokens of each group, one sign bit for each of the 17 real and
 * 15 imaginary independent coefficients, and the mean |Re|, mean |Im| over the
 * 32 bins as fp16 scales.  `channel_metric` and `use_fft` in the parameters
 * select the paper's other ranking metrics and its non-FFT 1-bit code.
 *   K_dev        in : [L, B, Hkv, Tq, 128] fp16
 *   packed_K_dev out: >= vidkv_packed_keys_bytes(params) bytes
 *   workspace_dev   : >= vidkv_workspace_bytes(params, 0) bytes, scratch     */
vidkv_status vidkv_quantize_keys(const vidkv_params *params, const void *K_dev,
                                 void *packed_K_dev, size_t packed_bytes,
                                 void *workspace_dev, size_t workspace_bytes,
                                 void *hip_stream);

/* Alg. 2 (1.58Quant with token protection): per channel and 32-token group
 * s = mean |V| over the unprotected tokens, code = +1 / -1 / 0 against
 * +-gamma*s (Eq. 6); protected tokens are coded 0 and their rows copied
 * verbatim.  The protected set is shared by all layers and heads of a
 * sequence and is given either as scores (top n_salient, ties: lower index
 * first; Eq. 7 scores are computed by the caller) or as an index list.
 *   V_dev           in : [L, B, Hkv, Tq, 128] fp16
 *   saliency_dev    in : [B, Tq] float32, or NULL
 *   salient_idx_dev in : [B, n_salient] int32, strictly ascending per
 *                        sequence, or NULL.  With n_salient > 0 exactly one of
 *                        the two is non-NULL; with n_salient == 0 both are
 *                        ignored.  Entries outside 0..Tq-1 and repeated
 *                        entries are not an error: they are dropped, fewer
 *                        tokens are protected (with salient_bits == 2 the
 *                        statistics of the last group of protected rows are
 *                        then unspecified).
 *   packed_V_dev    out: >= vidkv_packed_values_bytes(params) bytes
 *   workspace_dev      : >= vidkv_workspace_bytes(params, 1) bytes           */
vidkv_status vidkv_quantize_values(const vidkv_params *params, const void *V_dev,
                                   const float *saliency_dev,
                                   const int32_t *salient_idx_dev,
                                   void *packed_V_dev, size_t packed_bytes,
                                   void *workspace_dev, size_t workspace_bytes,
                                   void *hip_stream);

/* Alg. 3 and Alg. 2 on the K and V tensors of the same tokens in one call (the
 * compression step at the end of Alg. 1, Prefill): the packed buffers come out
 * byte-identical to vidkv_quantize_keys followed by vidkv_quantize_values.
 * Sequences of up to 32768 tokens run in line, in two launches (few groups) or
 * three with the range metric (more with the two others, and with some 33000
 * heads or more).
 * For longer ones the protected-token selection is a chain of short dependent
 * launches; with a side stream it is enqueued there so that it runs beside the key
 * passes (only when the key tensor is 96 MiB or more; smaller inputs run in
 * line), and joined back before the value coding pass.
 * Arguments as for the two separate calls;
 *   workspace_dev : >= vidkv_workspace_bytes(params, 3) bytes
 *   side          : NULL, or the caller's side stream and events (all three
 *                   handles non-NULL, and where the call uses it, the stream
 *                   on the current device, else VIDKV_EINVAL)                 */
vidkv_status vidkv_quantize_kv(const vidkv_params *params, const void *K_dev,
                               const void *V_dev, const float *saliency_dev,
                               const int32_t *salient_idx_dev, void *packed_K_dev,
                               size_t packed_K_bytes, void *packed_V_dev,
                               size_t packed_V_bytes, void *workspace_dev,
                               size_t workspace_bytes, void *hip_stream,
                               const vidkv_side_stream *side);

/* Alg. 1, Decoding, for one layer: out = Softmax(scale * q [K'; K_r]^T) [V'; V_r]
 * (Eq. 3) where K', V' are the dequantized packed tokens (never materialised
 * in memory) and K_r, V_r the first tail_len[b] rows of the fp16 residual
 * buffers.  Appending the new token to the residual buffers and advancing
 * tail_len is the caller's job.
 *   layer           : 0..L-1, selects the layer inside the packed buffers
 *   q_dev        in : [B, Hq, 128] fp16
 *   packed_K_dev, packed_V_dev in : as written by the two quantize calls with
 *                     the same params
 *   K_tail_dev, V_tail_dev in : [B, Hkv, tail_capacity, 128] fp16 of this
 *                     layer; may be NULL when tail_capacity == 0
 *   tail_len_dev in : [B] int32, each 0..tail_capacity; NULL means all zero
 *   out_dev     out : [B, Hq, 128] fp16 (fp32 accumulation, RNE at the end)
 *   workspace_dev   : >= vidkv_workspace_bytes(params, 2) bytes (the size
 *                     depends on t_capacity, not on t_quant).  It holds the
 *                     finest split of the cache; earlier builds reported, and
 *                     this one still takes, the size of a coarser one, which
 *                     the call then uses
 * With Tq == 0 this is plain attention over the residual tokens; a sequence
 * with no token at all gets zeros.
 * Everything runs in line on `hip_stream`, with and without a side stream (a
 * large residual block no longer gains from one).
 *   side            : NULL, or a side stream and events (all three handles
 *                     non-NULL, else VIDKV_EINVAL): not used                 */
vidkv_status vidkv_decode_attention(const vidkv_params *params, int32_t layer,
                                    const void *q_dev, const void *packed_K_dev,
                                    const void *packed_V_dev, const void *K_tail_dev,
                                    const void *V_tail_dev, int32_t tail_capacity,
                                    const int32_t *tail_len_dev, void *out_dev,
                                    void *workspace_dev, size_t workspace_bytes,
                                    void *hip_stream, const vidkv_side_stream *side);

/* vidkv_decode_attention for callers that cannot allocate device memory or
 * carry a workspace: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, checks and result as
 * vidkv_decode_attention, without the workspace: the split partials go to a
 * device array inside the library's image, VIDKV_NOALLOC_SCRATCH_BYTES large,
 * which every GPU that runs the library holds until the process ends.  The
 * call allocates nothing and takes no side stream: all of its kernels, the
 * one for a large residual block included, run in line on `hip_stream`.
 * A shape whose partials (what vidkv_workspace_bytes(params, 2) reports) do
 * not fit the array returns VIDKV_ENOSPACE and launches nothing.  The device
 * address of the array is looked up at the first call on each device (make
 * that call outside a stream capture).  All calls on one GPU share the one
 * array: two such calls that may run at the same time - on different streams
 * of that GPU, or from different host threads - race and give wrong results;
 * calls ordered on one stream are fine.                                        */
#define VIDKV_NOALLOC_SCRATCH_BYTES (16u << 20)
vidkv_status vidkv_decode_attention_noalloc(const vidkv_params *params, int32_t layer,
                                            const void *q_dev, const void *packed_K_dev,
                                            const void *packed_V_dev, const void *K_tail_dev,
                                            const void *V_tail_dev, int32_t tail_capacity,
                                            const int32_t *tail_len_dev, void *out_dev,
                                            void *hip_stream);

/* Alg. 1, Decoding, the step taken when the residual buffers are full (R
 * tokens): the first n_flush residual tokens of every sequence of one layer
 * are coded and appended to the packed buffers as tokens t_quant ..
 * t_quant + n_flush - 1.  Values: Alg. 2's 1.58Quant without protected tokens
 * (Eq. 6).  Keys: the group coding of Alg. 3 (Eq. 4 / Eq. 5) with the channel
 * split chosen when the cache was first quantized - the ranking by range is
 * not repeated, and the groups already packed are not touched (re-coding their
 * dequantized values with the same split would reproduce them).
 *   params          : t_quant = tokens packed so far (> 0), t_capacity >=
 *                     t_quant + n_flush
 *   layer           : 0..L-1
 *   K_tail_dev, V_tail_dev in : [B, Hkv, tail_capacity, 128] fp16 of this layer;
 *                     rows 0..n_flush-1 of every head must be valid tokens
 *   n_flush         : multiple of 32, 0 < n_flush <= tail_capacity
 *   packed_K_dev, packed_V_dev in/out : as written by the quantize calls with
 *                     the same t_capacity
 * Afterwards the caller raises t_quant by n_flush - once every layer has been
 * flushed - and moves any remaining residual rows to the front.  No workspace. */
vidkv_status vidkv_flush_residual(const vidkv_params *params, int32_t layer,
                                  const void *K_tail_dev, const void *V_tail_dev,
                                  int32_t tail_capacity, int32_t n_flush,
                                  void *packed_K_dev, size_t packed_K_bytes,
                                  void *packed_V_dev, size_t packed_V_bytes,
                                  void *hip_stream);

/* Sec. 3.3 (2), Eq. 7: the cross-modal score I(i, j) = X_v(i) . X_t(j) between
 * visual token i and text token j, summed over the text tokens of the
 * sequence: scores[b][i] = sum_j X_v[b][i] . X_t[b][j] (fp32 accumulation).
 * The result is what vidkv_quantize_values takes as saliency_dev.  Which
 * hidden states to pass (the paper does not say which layer) is the caller's
 * choice.
 *   X_v_dev   in : [B, n_visual, hidden_dim] fp16, 16-byte aligned
 *   X_t_dev   in : [B, n_text, hidden_dim] fp16, n_text >= 1
 *   hidden_dim   : multiple of 8, 8..16384
 *   scores_dev out: [B, n_visual] float32
 *   workspace_dev: >= vidkv_saliency_workspace_bytes(B, hidden_dim) bytes      */
size_t vidkv_saliency_workspace_bytes(int32_t batch, int32_t hidden_dim);
vidkv_status vidkv_saliency_scores(const void *X_v_dev, const void *X_t_dev, int32_t batch,
                                   int32_t n_visual, int32_t n_text, int32_t hidden_dim,
                                   float *scores_dev, void *workspace_dev,
                                   size_t workspace_bytes, void *hip_stream);

/* ---- rotary positions and the 8-bit cache ------------------------------------
 * What stands beside the packed cache: rotary positions on several axes for the
 * queries and keys that go into either cache, and a cache that holds keys and
 * values in 8 bits with one magnitude for each block of 32 tokens and head, for
 * layers and streams that do not stand the packed one: written token by token or
 * in bulk, read back, and attended over by any number of queries.
 *
 * Tensors of these calls are views [B, heads, tokens, channels] with strides of
 * their own; the channels of a token lie next to each other.  `data` is 16-byte
 * aligned device memory and every stride a multiple of 16 bytes (else
 * VIDKV_EINVAL), so both [B, heads, tokens, D] and the transposed view of what a
 * projection leaves ([B, tokens, heads, D]) are taken as they are.  Outputs must
 * not overlap inputs unless stated, nor themselves.  */
typedef enum { VIDKV_F16 = 0, VIDKV_BF16 = 1, VIDKV_F32 = 2 } vidkv_dtype;

typedef struct vidkv_view {
  void *data;             /* device */
  int64_t stride_batch;   /* in elements */
  int64_t stride_head;
  int64_t stride_token;
  int32_t dtype;          /* vidkv_dtype */
} vidkv_view;

/* Rotary positions: pair i of a head's first rot_dim channels is turned by the
 * angle pos[axis[i]] * freq_i,
 *     y1 = x1 cos - x2 sin,   y2 = x2 cos + x1 sin;
 * the channels behind rot_dim are passed on.  Plain host data, made by
 * vidkv_rotary_init, never retained; `axis` and `turn` may be set by the caller
 * (an interleaved order of the axes, scaled frequencies). */
#define VIDKV_ROTARY_PAIRS 128
typedef struct vidkv_rotary {
  int32_t head_dim;       /* 16..256, multiple of 16                             */
  int32_t rot_dim;        /* 16..head_dim, multiple of 16                        */
  int32_t adjacent;       /* pair i is channels 0: i and i + rot_dim/2,
                             1: 2i and 2i + 1                                    */
  int32_t n_axes;         /* 1..4 rows of positions (time, height, width)        */
  uint8_t axis[VIDKV_ROTARY_PAIRS];  /* the row that pair i takes its position from */
  uint64_t turn[VIDKV_ROTARY_PAIRS]; /* freq_i as turns a position, times 2^64 (modulo
                             2^64): products with a position are exact, so angles of
                             far positions are as accurate as those of near ones */
} vidkv_rotary;

/* Host function: fills *rot.  sections[n_axes] (host) are the pairs of each axis,
 * in order, rot_dim / 2 in all.  freq_i = theta^(-2i / rot_dim) radians a position,
 * or freq[i] (host, rot_dim / 2 numbers) where that is not NULL. */
vidkv_status vidkv_rotary_init(vidkv_rotary *rot, int32_t head_dim, int32_t rot_dim,
                               int32_t adjacent, int32_t n_axes, const int32_t *sections,
                               double theta, const double *freq);

/* Rotates the queries and keys of the same tokens (either may be NULL).
 *   pos_dev     in : [n_axes, batch, n_tokens] int32, any values
 *   q, q_out       : [batch, n_q_heads, n_tokens, head_dim], same dtype; q_out
 *                    may be the same view as q
 *   k, k_out       : [batch, n_k_heads, ...] likewise, of q's dtype
 *   inverse        : 0 turns by +angle; 1 by -angle: undoes the rotation, and is
 *                    its backward pass (gradients of y in, gradients of x out)
 * Computed in fp32 (angles within the nearest quarter turn to 24 bits: 2^-28 turns,
 * at any position), rounded once.  batch * n_tokens is at most 2^26 (else
 * VIDKV_ESHAPE). */
vidkv_status vidkv_rotary_apply(const vidkv_rotary *rot, int32_t inverse, int32_t batch,
                                int32_t n_tokens, const int32_t *pos_dev, int32_t n_q_heads,
                                const vidkv_view *q, const vidkv_view *q_out, int32_t n_k_heads,
                                const vidkv_view *k, const vidkv_view *k_out, void *hip_stream);

/* Geometry of an 8-bit cache.  A block is 32 tokens of one head; for K and for V
 * it holds its magnitude A = max |x|, clamped to 2^-40..2^40, and codes
 *   code 0 (int8): rint(x * 127 / A), value = code * A / 127
 *   code 1 (e4m3): the nearest e4m3 number to x * 448 / A, value = that * A / 448
 * (ties to even in both; |x| beyond A = 2^40 has the largest code).  An infinity is
 * taken as its type's largest number, which like any number far above the others
 * leaves these few bits or none, tokens that the block held before among them; a
 * NaN is taken as zero. */
typedef struct vidkv_cache8 {
  int32_t n_layers, batch, n_kv_heads;
  int32_t n_q_heads;      /* multiple of n_kv_heads, any ratio                   */
  int32_t head_dim;       /* must be 128                                         */
  int32_t capacity;       /* tokens a sequence, multiple of 32, 32..2^28         */
  int32_t code;           /* 0 int8, 1 e4m3                                      */
  float softmax_scale;    /* multiplies q.k before the softmax, > 0              */
} vidkv_cache8;

/* Size queries (host): bytes of the cache buffer of all layers, and of the
 * workspace that is enough for attention calls of up to n_query queries a
 * sequence; 0 when *p or n_query is invalid.  n_kv_heads and batch at most
 * 65535; at most 2^28 tokens a call, and 2^28 queries times heads of a group
 * (VIDKV_ESHAPE). */
size_t vidkv_cache8_bytes(const vidkv_cache8 *p);
size_t vidkv_cache8_workspace_bytes(const vidkv_cache8 *p, int32_t n_query);

/* Codes the first count[b] of n_tokens new tokens of one layer as tokens
 * start[b], start[b] + 1, ... of sequence b.  Tokens from start[b] on that the
 * cache held before are given up.  A block that begins before start[b] keeps its
 * live tokens: where the new ones raise its magnitude from A to A', their codes c
 * become the code of value(c) (in the code's units) * A / A'; else they are not
 * touched (those tokens have to have been written, or the buffer cleared).  Codes
 * behind the last new token are left as they were.
 *   K, V      in : [B, Hkv, n_tokens, 128], fp16 or bf16, both the same dtype;
 *                  rows from count[b] on are not read
 *   start_dev in : [B] int32; a negative start writes nothing for the sequence,
 *                  tokens behind the capacity are dropped
 *   count_dev in : [B] int32 (values beyond 0..n_tokens are taken as the nearer
 *                  end), or NULL: n_tokens of every sequence
 *   rot, pos_dev : both NULL, or the rotation of the keys (head_dim 128) with the
 *                  positions [n_axes, B, n_tokens] of the new tokens: the cache is
 *                  the same as after vidkv_rotary_apply on K
 *   cache_dev in/out: >= vidkv_cache8_bytes(p) bytes, 256-byte aligned, need not
 *                  be cleared before its first use                              */
vidkv_status vidkv_cache8_write(const vidkv_cache8 *p, int32_t layer, int32_t n_tokens,
                                const vidkv_view *K, const vidkv_view *V,
                                const int32_t *start_dev, const int32_t *count_dev,
                                const vidkv_rotary *rot, const int32_t *pos_dev,
                                void *cache_dev, size_t cache_bytes, void *hip_stream);

/* Reads tokens start[b] .. start[b] + n_tokens - 1 of one layer back as values
 * (fp16, bf16 or fp32; either output may be NULL).  Tokens outside
 * 0..capacity-1 come as zeros; those never written are unspecified, or zeros where
 * the buffer was cleared. */
vidkv_status vidkv_cache8_read(const vidkv_cache8 *p, int32_t layer, int32_t n_tokens,
                               const int32_t *start_dev, const void *cache_dev,
                               size_t cache_bytes, const vidkv_view *K, const vidkv_view *V,
                               void *hip_stream);

/* out = Softmax(scale * q K'^T) V' over the first length[b] tokens of one layer.
 * The queries are the last ones of the sequence: query i of q_count[b] stands at
 * token length[b] - q_count[b] + i and, with causal = 1, sees the tokens up to
 * itself; with causal = 0 all.  A query that sees no token, and the rows from
 * q_count[b] on, get zeros.  Scores scale * q.k are held in fp32: a weight's
 * relative error is some 2^-24 of the largest of them (which is why they are to
 * stay below 2^24; beyond, weights are unspecified).  Weights are multiplied with
 * the values in 11 bits, each rounded by at most 2^-11 of itself, and the sum that
 * they are divided by is that of the rounded ones: equal values come out as they
 * are, others to 2^-10 of Softmax(..) |V'| at most.  (Weights in a block whose values
 * are an eighth of those of others or less are summed as they are.)
 * Tokens that were never written are unspecified, as in reading, but in a cleared
 * buffer they are zeros (a sequence padded on the left), and take part as such.
 *   q         in : [B, Hq, n_query, 128], fp16 or bf16 (the elements of a bf16 row
 *                  are taken to 2^-39 of its largest)
 *   out      out : likewise, of q's dtype (fp32 accumulation)
 *   length_dev in: [B] int32, taken as 0..capacity
 *   q_count_dev in: [B] int32, taken as 0..n_query; NULL: n_query
 *   workspace_dev : >= vidkv_cache8_workspace_bytes(p, n_query) bytes, 256-byte
 *                   aligned                                                     */
vidkv_status vidkv_cache8_attention(const vidkv_cache8 *p, int32_t layer, int32_t n_query,
                                    int32_t causal, const vidkv_view *q, const void *cache_dev,
                                    size_t cache_bytes, const int32_t *length_dev,
                                    const int32_t *q_count_dev, const vidkv_view *out,
                                    void *workspace_dev, size_t workspace_bytes,
                                    void *hip_stream);

/* ---- trees of drafted tokens --------------------------------------------------
 * Checking several drafted tokens in one step of the target model.  Node 0 of a
 * sequence's tree is the last token that was sampled, whose successor is asked for;
 * node i > 0 is a drafted token behind node parent[i] < i.  The nodes' keys and
 * values stay in 16 bits beside the 8-bit cache - a token that is turned down would
 * leave its magnitude in a block's codes - and those that stand are appended to it:
 *   once a step       vidkv_tree_masks: what each node sees, and its position
 *   in every layer    vidkv_rotary_apply, vidkv_cache8_tree_attention
 *   once a step       vidkv_tree_verify, vidkv_cache8_append_path (all layers)
 * A tree has 1..VIDKV_TREE_NODES nodes; count_dev[b] (taken as 0..n_nodes, NULL:
 * n_nodes) says how many of them sequence b has.                                */
#define VIDKV_TREE_NODES 256
#define VIDKV_TREE_VOCAB (1 << 22)

/* Masks and positions.  A node sees itself and its ancestors.
 *   parent_dev in : [B, n_nodes] int32; -1 or anything else outside 0..i-1: node i
 *                   has no ancestors.  NULL: a chain, node i is behind node i - 1
 *   mask_dev  out : [B, n_nodes, ceil(n_nodes / 64)] uint64: bit j % 64 of word
 *                   j / 64 of node i: it sees node j.  None for nodes from count on
 *   pos_dev   out : [n_axes, B, n_nodes] int32 as vidkv_rotary_apply takes them,
 *                   n_axes 1..4: base_dev[b] and the node's ancestors in number on
 *                   every axis (base from count on); both NULL: none             */
vidkv_status vidkv_tree_masks(int32_t batch, int32_t n_nodes, const int32_t *parent_dev,
                              const int32_t *count_dev, uint64_t *mask_dev, int32_t n_axes,
                              const int32_t *base_dev, int32_t *pos_dev, void *hip_stream);

/* out_i = Softmax(scale * q_i [K'; K]^T) [V'; V]: the first length[b] tokens of one
 * layer of the cache, and the nodes that mask i has, of count[b] there are (any mask: its bits
 * from count on are not looked at).  A node without any and the rows from count[b]
 * on get zeros.  K and V are taken as the cache takes them where they leave its range
 * (an infinity as its type's largest number, a NaN as zero, bf16 held to 2^40),
 * else as they are; their rows from count[b] on are not read.  Precision as
 * vidkv_cache8_attention.
 *   q, out, K, V   : [B, Hq, n_nodes, 128] and [B, Hkv, n_nodes, 128], all fp16 or
 *                    all bf16
 *   mask_dev    in : [B, n_nodes, ceil(n_nodes / 64)] uint64, 8-byte aligned
 *   workspace_dev  : >= vidkv_cache8_workspace_bytes(p, n_nodes) bytes; the order of
 *                    sums does not depend on what more it holds                   */
vidkv_status vidkv_cache8_tree_attention(const vidkv_cache8 *p, int32_t layer, int32_t n_nodes,
                                         const vidkv_view *q, const vidkv_view *K,
                                         const vidkv_view *V, const uint64_t *mask_dev,
                                         const void *cache_dev, size_t cache_bytes,
                                         const int32_t *length_dev, const int32_t *count_dev,
                                         const vidkv_view *out, void *workspace_dev,
                                         size_t workspace_bytes, void *hip_stream);

/* Rows of probabilities, [B, n_nodes, vocab]: a row's entries lie next to each other, rows
 * wherever their elements are aligned. */
typedef struct vidkv_rows {
  const void *data;       /* device */
  int64_t stride_batch;   /* in elements */
  int64_t stride_row;
  int32_t dtype;          /* vidkv_dtype, fp32, fp16 or bf16 */
} vidkv_rows;

/* Which drafted tokens stand, and the token behind them, so that what comes out is
 * distributed as if it were sampled from the target model token by token.  From node 0
 * on, the children of the node reached are tried in order; R is what is left of target
 * row u of that node, taken to sum to one.
 *   draft NULL        the drafted tokens are no random ones.  Token x of child i
 *                     stands if uniform[i] < R(x); else R(x) becomes 0
 *   draft, distinct 0 each child was drawn from row u of draft, Q: x stands if
 *                     uniform[i] Q(x) < R(x); else R becomes max(R - Q, 0)
 *   draft, distinct 1 children were drawn without putting back: likewise, and Q(x)
 *                     becomes 0 and Q is divided by 1 less the row's probability of the
 *                     tokens turned down; where that is not above 0 there is nothing that
 *                     a further child could have come from, and none is tried
 * and R is divided by its sum.  The walk goes on at a child that stands, with its rows,
 * and ends where no child does.  The next token is the first v with
 * sum_{w <= v} R(w) > uniform[0] sum R (the last with R(v) > 0 if there is none).
 * Without draft, and with distinct, a token that an earlier sibling had is passed over;
 * one outside 0..vocab-1 always is.  Where nothing at all would be left of R (with numbers
 * in [0, 1): by rounding alone), with draft it stays what it was and no further child is
 * tried, without it is the target's row again.
 * All rows are taken to sum to one, as float32 rows of a softmax do to some 2^-20.  A draft
 * row that sums to 1 + e puts |e| of a token's probability off, and with distinct
 * |e| / (1 + e - t) behind tokens turned down that have t of the row: nothing is promised of
 * distinct rows whose rounding is not small against 1 - t.  In 16 bits |e| is up to 2^-8
 * (bf16) or 2^-11 and 2^-25 for each entry below 2^-14 (fp16), and t soon 0.99; where that
 * matters, make such rows float32, divide them by their sums, and both draw from them and
 * pass them.
 * Sums and decisions are in 64 bits.  Entries have to be finite; those not above 0 count
 * as 0.
 *   target     in : probabilities behind each node.  draft: of target's dtype
 *   token_dev  in : [B, n_nodes] int32 (node 0's is not looked at)
 *   parent_dev in : [B, n_nodes] int32; outside 0..i-1: node i is no child.  NULL: a chain
 *   uniform_dev in: [B, n_nodes] float32, independent numbers in [0, 1)
 *   path_dev  out : [B, n_nodes] int32: node 0 and the nodes that stand, then -1
 *   accepted_dev out: [B] int32: the nodes of the path, 1 at least (0 where count[b] is 0)
 *   next_dev  out : [B] int32: the next token; -1 where count[b] is 0 or the last
 *                   node's row has nothing above 0
 *   workspace_dev : >= vidkv_tree_verify_workspace_bytes(..) bytes, 256-byte aligned
 * The size query gives 0 for sizes outside 1..65535, 1..VIDKV_TREE_NODES and
 * 1..VIDKV_TREE_VOCAB (the call: VIDKV_ESHAPE). */
size_t vidkv_tree_verify_workspace_bytes(int32_t batch, int32_t n_nodes, int32_t vocab);
vidkv_status vidkv_tree_verify(int32_t batch, int32_t n_nodes, int32_t vocab,
                               const vidkv_rows *target, const vidkv_rows *draft, int32_t distinct,
                               const int32_t *token_dev, const int32_t *parent_dev,
                               const int32_t *count_dev, const float *uniform_dev,
                               int32_t *path_dev, int32_t *accepted_dev, int32_t *next_dev,
                               void *workspace_dev, size_t workspace_bytes, void *hip_stream);

/* Appends nodes path[b][0 .. accepted[b] - 1] of all layers as tokens start[b],
 * start[b] + 1, ..., the same as vidkv_cache8_write of those rows in every layer
 * would.  K and V are those of layer 0; layer l's are l * k_stride_layer (V: v_stride_layer)
 * elements further on.  Heads of all sequences and layers are fewer than 2^24 (else
 * VIDKV_ESHAPE).
 *   K, V        in : [B, Hkv, n_nodes, 128], fp16 or bf16, both the same dtype, turned already
 *   path_dev    in : [B, n_nodes] int32, as vidkv_tree_verify leaves it: any nodes
 *                    in any order; the path ends before an entry outside 0..n_nodes-1
 *   accepted_dev in: [B] int32 (taken as 0..n_nodes)
 *   start_dev   in : [B] int32; negative: nothing is written; tokens behind the capacity
 *                    are dropped                                                   */
vidkv_status vidkv_cache8_append_path(const vidkv_cache8 *p, int32_t n_nodes, const vidkv_view *K,
                                      int64_t k_stride_layer, const vidkv_view *V,
                                      int64_t v_stride_layer, const int32_t *path_dev,
                                      const int32_t *accepted_dev, const int32_t *start_dev,
                                      void *cache_dev, size_t cache_bytes, void *hip_stream);

/* Measurement aids, not part of the method.  Each takes the arguments of the
 * entry point it is named after, checks them the same way, and launches only
 * the kernels selected by `stages`, so that a benchmark can bracket a single
 * kernel with events.  The buffers must already hold what the skipped kernels
 * would have written (run the full entry point once first).
 *   quantize_keys   : bit 0 per-channel min/max over all tokens (Alg. 3, range)
 *                     bit 1 top-n_anom channel selection
 *                     bit 2 per-group coding pass (Eq. 4 and Eq. 5)
 *   quantize_values : bit 0 protected-token selection, bit 1 ternary coding pass
 *   decode_attention: bit 0 split-T partial attention, bit 1 merge              */
vidkv_status vidkv_quantize_keys_stages(const vidkv_params *params, const void *K_dev,
                                        void *packed_K_dev, size_t packed_bytes,
                                        void *workspace_dev, size_t workspace_bytes,
                                        uint32_t stages, void *hip_stream);
vidkv_status vidkv_quantize_values_stages(const vidkv_params *params, const void *V_dev,
                                          const float *saliency_dev,
                                          const int32_t *salient_idx_dev, void *packed_V_dev,
                                          size_t packed_bytes, void *workspace_dev,
                                          size_t workspace_bytes, uint32_t stages,
                                          void *hip_stream);
vidkv_status vidkv_decode_attention_stages(const vidkv_params *params, int32_t layer,
                                           const void *q_dev, const void *packed_K_dev,
                                           const void *packed_V_dev, const void *K_tail_dev,
                                           const void *V_tail_dev, int32_t tail_capacity,
                                           const int32_t *tail_len_dev, void *out_dev,
                                           void *workspace_dev, size_t workspace_bytes,
                                           uint32_t stages, void *hip_stream,
                                           const vidkv_side_stream *side);

/* Measurement aid, not part of the method: dst[i] = src[i] for `bytes` bytes
 * (multiple of 16, both 16-byte aligned) with the library's streaming access
 * pattern; used to calibrate hardware byte counters and the achievable HBM
 * rate. */
vidkv_status vidkv_calib_copy(void *dst_dev, const void *src_dev, size_t bytes,
                              void *hip_stream);

const char *vidkv_status_string(vidkv_status status);
int vidkv_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* VIDKV_H */
