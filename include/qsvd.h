/*
 * qsvd.h -- C ABI of the QSVD latent-QKV hot path on AMD Instinct MI355X (gfx950).
 *
 * QSVD ("Efficient Low-rank Approximation for Unified Query-Key-Value Weight
 * Compression in Low-Precision Vision-Language Models", arXiv 2510.16292)
 * replaces the three projections W_q, W_k, W_v of an attention layer by one
 * joint truncated SVD of [W_q | W_k | W_v] (Section 3.1, Eq. 2-4): a shared
 * down-projection W^d (d x r) and an up-projection W^u = [W^u_q | W^u_k | W^u_v]
 * (r x N).  The per-token latent C = X W^d is the only thing cached
 * (Section 3.1); keys and values are rebuilt from it, K = C W^u_k and
 * V = C W^u_v (Eq. 5).  Weights and activations are quantized (Section 3.3,
 * Eq. 11-12; per-token symmetric activations and round-to-nearest
 * per-channel symmetric weights, Section 4).
 *
 * Conventions for every call:
 *  - Pointers marked "device" are device (HBM) addresses allocated by the
 *    caller; the library never allocates, frees or keeps device memory, and
 *    keeps no state between calls except the optional profiler.
 *  - `stream` is a hipStream_t (NULL = the null stream).  Calls enqueue work
 *    on it and return without synchronizing.
 *  - Arguments are validated on the host before any GPU work is enqueued.  On
 *    any status other than QSVD_OK nothing was enqueued, outputs are left
 *    untouched and cache state (seq_len, max_len) is unchanged -- except
 *    QSVD_ERR_HIP, which reports a failed launch after validation passed.
 *    qsvd_last_error() describes the most recent failure of the calling thread.
 *  - Row-major layouts; "[a][b]" means b is the contiguous index.
 *  - Integer codes are symmetric two's complement: int8 in [-127, 127], int4
 *    in [-7, 7] packed two per byte, element 2i in the low nibble of byte i.
 */
#ifndef QSVD_H
#define QSVD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  QSVD_OK = 0,
  QSVD_ERR_INVALID_ARG = 1,  /* null pointer, negative size, inconsistent shapes */
  QSVD_ERR_UNSUPPORTED = 2,  /* well-formed but outside what the kernels implement */
  QSVD_ERR_CAPACITY = 3,     /* an append would exceed the cache capacity */
  QSVD_ERR_WORKSPACE = 4,    /* workspace missing or smaller than the size query */
  QSVD_ERR_HIP = 5           /* a HIP runtime call or kernel launch failed */
} qsvd_status;

/* Latent cache storage formats. */
enum { QSVD_CACHE_F16 = 0, QSVD_CACHE_I8 = 1, QSVD_CACHE_I4 = 2 };

/* Decode attention forms.  RECONSTRUCT rebuilds K and V from the latent for
 * every cached token (Eq. 5) and attends as usual; ABSORBED folds W^u_k into
 * the query and applies W^u_v after the latent-space weighted sum (the
 * latent-attention form of Section 1 and 2.2).  Both compute the same
 * attention; AUTO picks the faster one for the layer (ABSORBED). */
enum { QSVD_ATTN_AUTO = 0, QSVD_ATTN_ABSORBED = 1, QSVD_ATTN_RECONSTRUCT = 2 };

/* 16-bit element types of the layer operators. */
enum { QSVD_F16 = 0, QSVD_BF16 = 1 };

/* Which up-projection outputs qsvd_lowrank_qkv_prefill writes. */
enum { QSVD_OUT_Q = 1, QSVD_OUT_K = 2, QSVD_OUT_V = 4 };

/* One attention layer after the offline stage (joint SVD, truncation, beta
 * split, weight quantization).  N = (n_q_heads + 2 * n_kv_heads) * head_dim.
 * Query head h reads key/value head floor(h * n_kv_heads / n_q_heads). */
typedef struct {
  int32_t d;           /* embedding dimension E (contraction of X W^d) */
  int32_t r;           /* joint rank */
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t w_bits;      /* 8: int8 codes; 4: packed int4 codes */
  int32_t w_group;     /* 0: one scale per output channel; G > 0: one scale per
                          output channel and per G contraction rows */
  const void*  a_t;    /* device, W^d codes transposed: [r][d] int8 or [r][d/2] int4 */
  const float* s_a;    /* device, W^d scales: [r] (w_group 0) or [d/G][r] */
  const void*  b_t;    /* device, W^u codes transposed: [N][r] int8 or [N][r/2] int4;
                          rows 0..Hq*hd-1 are W^u_q, then W^u_k, then W^u_v */
  const float* s_b;    /* device, W^u scales: [N] (w_group 0) or [r/G][N] */
} qsvd_layer;

/* Latent cache of `batch` sequences.  Sequence b holds seq_len[b] rows.
 * F16: data is [batch][capacity][r] fp16, scale NULL.
 * I8:  data is [batch][capacity][r] int8, scale [batch][capacity] fp32.
 * I4:  data is [batch][capacity][r/2] packed int4, scale [batch][capacity] fp32.
 * A row of an integer cache is Q(C) of the token (its codes and scale). */
typedef struct {
  int32_t  fmt;        /* QSVD_CACHE_* */
  int32_t  batch;
  int32_t  capacity;   /* rows per sequence */
  int32_t  r;
  void*    data;       /* device */
  float*   scale;      /* device or NULL (F16) */
  int32_t* seq_len;    /* device [batch] */
  int32_t  max_len;    /* host: an upper bound of every seq_len[b]; the caller sets
                          it when initialising seq_len, append advances it */
  int32_t* overflow;   /* device, optional (NULL: not reported): an append that finds
                          seq_len[b] + n_new > capacity on the device (possible only
                          when the host check was bypassed, e.g. by a graph replay)
                          stores 1 here; the caller clears it */
} qsvd_cache;

/* Per-token symmetric activation quantization (Section 4 setup; Q(.) of Eq. 12).
 * Per row m, in fp32: a = clip * max_k |x[m][k]|; if a == 0 then s = 1 and all
 * codes are 0, else inv = Qm / a (IEEE division), s = a / Qm and
 * q = clamp(rint(x * inv), -Qm, Qm) with ties to even; Qm = 2^(bits-1) - 1.
 *   x   device fp16 [M][ldx] (first K columns used)
 *   xq  device int8 [M][K] (bits 8) or packed int4 [M][K/2] (bits 4)
 *   sx  device fp32 [M]
 * Requires K % 8 == 0, ldx % 8 == 0, 16-byte aligned x; bits 8 or 4; 0 < clip <= 1. */
qsvd_status qsvd_quantize_act(const void* x, int64_t M, int32_t K, int64_t ldx, int32_t bits,
                              float clip, void* xq, float* sx, void* stream);

/* Per-token quantization of rotated activations, Q(X H1^T) (Eq. 11-12), for
 * layers whose input rotation H1 cannot be folded into the previous layer;
 * the layer's W^d then holds H1 W^d (folded offline).
 *   H1 = blockdiag(H_B, ..., H_B) diag(signs) / sqrt(B), H_B the Sylvester
 *   Hadamard matrix of order B = block, so X H1^T = (X o signs) blockdiag(H_B) / sqrt(B).
 * Per row, in fp32: v_k = x_k * signs_k; the Walsh-Hadamard stages
 * h = 1, 2, 4, ..., B/2 in that order, each replacing (v_i, v_{i+h}) by
 * (v_i + v_{i+h}, v_i - v_{i+h}) for every i whose bit h is clear (each sum
 * rounded to fp32); y = v * c with c = fp32(1 / sqrt(B)); then y goes through
 * the quantizer of qsvd_quantize_act (same clip, scale and codes).
 *   x      device fp16 [M][ldx] (first K columns used)
 *   signs  device int8 [K] of +1 / -1 (NULL: all +1)
 *   block  B: a power of two >= 8 dividing K
 *   xq, sx as for qsvd_quantize_act
 * Requires K % 8 == 0, K <= 16384, ldx % 8 == 0, 16-byte aligned x, 8-byte
 * aligned xq and signs; bits 8 or 4; 0 < clip <= 1. */
qsvd_status qsvd_quantize_act_rotated(const void* x, int64_t M, int32_t K, int64_t ldx, int32_t bits,
                                      float clip, const int8_t* signs, int32_t block, void* xq,
                                      float* sx, void* stream);

/* Quantized joint low-rank QKV projection (Section 3.1 and Eq. 11-12):
 *   C   = (xq W^d codes) dequantized: fp32 (acc * sx[m]) * s_a[j] (per group:
 *         sum over groups of acc_g * s_a[g][j], then * sx[m]), stored as fp16
 *   Q(C) = per-token quantization of the fp16 C with act_bits (as qsvd_quantize_act, clip 1)
 *   [Q|K|V] = (Q(C) W^u codes) dequantized the same way, stored as fp16
 *   w        layer (host struct, device pointers)
 *   xq, sx   device, output of qsvd_quantize_act with act_bits, M rows
 *   c_h      device fp16 [M][r]                     (always written)
 *   cq, sc   device int8 [M][r] (or int4 [M][r/2]) and fp32 [M]   (always written)
 *   q, k, v  device fp16 [M][Hq*hd], [M][Hkv*hd], [M][Hkv*hd]; written when the
 *            matching QSVD_OUT_* bit is set (others may be NULL)
 *   dbg_acc_xa, dbg_acc_cb  optional device int32 [M][r] and [M][N] copies of
 *            the integer accumulators (w_group 0 only; NULL to skip)
 *   ws       unused (qsvd_prefill_workspace_size() returns 0; kept for callers
 *            that size one anyway)
 * Requires d % 64 == 0, r % 64 == 0, act_bits 8 or 4, int8 or int4 weights
 * with per-channel or per-group scales (groups a multiple of 64 dividing d and
 * r), 16-byte aligned xq, c_h, cq and weight codes.  More than 32 tokens also
 * need head_dim a multiple of 8 and 16-byte aligned q, k, v.  The integer
 * accumulator dumps need act_bits 8 and per-channel weights.  Other
 * combinations return QSVD_ERR_UNSUPPORTED. */
qsvd_status qsvd_lowrank_qkv_prefill(const qsvd_layer* w, const void* xq, const float* sx,
                                     int64_t M, int32_t act_bits, uint32_t out_mask,
                                     void* c_h, void* cq, float* sc, void* q, void* k, void* v,
                                     int32_t* dbg_acc_xa, int32_t* dbg_acc_cb,
                                     void* ws, size_t ws_bytes, void* stream);

size_t qsvd_prefill_workspace_size(const qsvd_layer* w, int64_t M, uint32_t out_mask);

/* Append n_new latent rows to every sequence of the cache (only C is buffered,
 * Section 3.1).  Source rows are token-major with sequence b's rows at
 * [b * n_new, (b + 1) * n_new):
 *   F16 cache: c_h  device fp16 [batch * n_new][r]           (cq, sc ignored)
 *   I8 / I4:   cq   device int8 [..][r] / int4 [..][r/2], sc device fp32 [..]
 * Row i of sequence b goes to position seq_len[b] + i; then seq_len[b] += n_new
 * on the device and c->max_len += n_new on the host.  Returns QSVD_ERR_CAPACITY
 * if c->max_len + n_new > c->capacity.  On the device, rows that would land at
 * or past capacity are not written, seq_len[b] stops at capacity and
 * *c->overflow is set to 1 (when given): a replayed graph, which skips the
 * host check, cannot grow a sequence past its buffer. */
qsvd_status qsvd_latent_cache_append(qsvd_cache* c, const void* c_h, const void* cq,
                                     const float* sc, int32_t n_new, void* stream);

/* One decode step's projection of the new tokens together with the append of
 * their latent rows (Section 3.1: one new token per sequence; only C is
 * buffered): per-token quantization of x with act_bits and clip, C = the
 * quantized down-projection, Q(C), the Q up-projection, and the append of each
 * sequence's latent row (fp16 C, or Q(C) codes and scale for an integer
 * cache) at position seq_len[b], then seq_len[b] += 1 on the device and
 * c->max_len += 1 on the host.  Every output byte, cache byte and length is
 * the one of qsvd_quantize_act + qsvd_lowrank_qkv_prefill(out_mask QSVD_OUT_Q)
 * + qsvd_latent_cache_append(n_new 1); the quantizer runs inside the
 * down-projection and the append inside the two products, so the step takes
 * two launches instead of four.
 *   x         device fp16 [batch][ldx], row b the new token of sequence b
 *   xq, sx    device outputs: Q(x) codes ([batch][d] int8 or [batch][d/2] int4) and scales
 *   c_h       device fp16 [batch][r]; cq, sc: Q(C) ([batch][r] / [batch][r/2], [batch])
 *   q         device fp16 [batch][Hq*hd]
 * Requires batch <= 32, an I8 cache with act_bits 8 or an I4 cache with
 * act_bits 4 (any act_bits for F16), ldx % 8 == 0, 16-byte aligned x, xq,
 * c_h, cq and weight codes, and the layer requirements of
 * qsvd_lowrank_qkv_prefill.  QSVD_ERR_CAPACITY if c->max_len + 1 > capacity;
 * on the device, a row at or past capacity is dropped as in
 * qsvd_latent_cache_append. */
qsvd_status qsvd_decode_project_append(const qsvd_layer* w, qsvd_cache* c, const void* x, int64_t ldx,
                                       int32_t act_bits, float clip, void* xq, float* sx, void* c_h,
                                       void* cq, float* sc, void* q, void* stream);

/* Causal self-attention of a prefill block over its own projections (Section
 * 3.1: in prefill every prompt token's keys and values are at hand as the rows
 * K = C W^u_k and V = C W^u_v that qsvd_lowrank_qkv_prefill wrote, Eq. 5 and
 * Eq. 11).  Token i of a sequence attends to tokens 0..i of the same sequence:
 * softmax(q k^T * sm_scale) v with an fp32 softmax, query head h reading
 * key/value head floor(h * n_kv_heads / n_q_heads).
 *   q           device fp16 [M][n_q_heads * head_dim] (the projection's Q)
 *   k, v        device fp16 [M][n_kv_heads * head_dim] (its K and V)
 *   cu_seqlens  device int32 [batch + 1]: sequence b is rows
 *               [cu_seqlens[b], cu_seqlens[b + 1]); nondecreasing, cu_seqlens[0] = 0
 *   max_seqlen  host: at least every sequence's length (sizes the launch)
 *   sm_scale    0 selects 1/sqrt(head_dim)
 *   out         device fp16 [M][n_q_heads * head_dim]
 * Requires head_dim 64 or 128 and 16-byte aligned q, k, v, out.  Rows of a
 * sequence longer than max_seqlen past max_seqlen are left unwritten.  No
 * workspace; asynchronous on `stream`. */
qsvd_status qsvd_prefill_attention(const void* q, const void* k, const void* v, int32_t batch,
                                   const int32_t* cu_seqlens, int32_t max_seqlen, int32_t n_q_heads,
                                   int32_t n_kv_heads, int32_t head_dim, float sm_scale, void* out,
                                   void* stream);

/* qsvd_prefill_attention for layers that apply a rotary position embedding
 * to q and k (the paper's layers have none; the position-encoded variant of
 * the same prefill step, with the same rotation as
 * qsvd_latent_decode_attention_rope).  Before the product, row i of a
 * sequence (its position within that sequence, counted from 0) has the pairs
 * (j, j + head_dim/2), j < head_dim/2, of every query and key head vector
 * turned by the angle i * rope_theta^(-2j/head_dim): the angle is formed in
 * revolutions and reduced to [0, 1) in fp64, its sine and cosine taken in
 * fp32, and the turned rows rounded to fp16 before the products.  Values are
 * not turned.  A decode step that continues the sequence over its cache sees
 * the same key positions.  Same arguments, requirements and errors as
 * qsvd_prefill_attention; rope_theta must be finite and > 1
 * (QSVD_ERR_INVALID_ARG otherwise). */
qsvd_status qsvd_prefill_attention_rope(const void* q, const void* k, const void* v, int32_t batch,
                                        const int32_t* cu_seqlens, int32_t max_seqlen, int32_t n_q_heads,
                                        int32_t n_kv_heads, int32_t head_dim, float sm_scale, float rope_theta,
                                        void* out, void* stream);

/* Attention of the newest queries of every sequence over its cached latent
 * rows (Section 3.1; decoding is l = 1): keys and values are C W^u_k and
 * C W^u_v of the stored rows (dequantized), softmax(q K^T * sm_scale) V with an
 * fp32 softmax.  The q_len queries of sequence b are its last q_len cached
 * positions (append first, then attend): query i sees positions
 * [0, seq_len[b] - q_len + i], causally.  A query with no visible position
 * (seq_len[b] < q_len - i) gets zeros.
 *   q     device fp16 [batch][q_len][Hq*hd] (the Q output of the projection)
 *   out   device fp16 [batch][q_len][Hq*hd]
 *   mode  QSVD_ATTN_ABSORBED (latent form), QSVD_ATTN_RECONSTRUCT (K, V
 *         rebuilt per cached token) or QSVD_ATTN_AUTO (absorbed when its shape
 *         is supported)
 *   sm_scale  0 selects 1/sqrt(head_dim)
 *   ws    device workspace of at least qsvd_decode_workspace_size() bytes
 * Requires head_dim % 32 == 0 and <= 128, batch <= 64, q_len <= max_len,
 * w_group 0 or a multiple of 64, 16-byte aligned q, out and s_b (else
 * QSVD_ERR_UNSUPPORTED or QSVD_ERR_INVALID_ARG).  The absorbed form takes
 * n_q_heads <= 64, r in {128, 512, 1024, 1536} (with at most 32 heads) or r
 * a multiple of 128 up to 3072, any cache format, and
 * batch * q_len * ceil(n_q_heads / 16) <= 65535 (batch * q_len <= 65535
 * with 32-head blocks).  The reconstruct form takes n_q_heads <= 64,
 * capacity <= 16384 and any cache format (F16 rows rebuild on the fp16
 * products, I8 on the int8 products, I4 on the 4-bit products), and with
 * q_len > 1 (causal attention of the last q_len positions over the rebuilt
 * rows on the fp16 matrix cores) head_dim 64 or 128.
 * The absorbed form sums a sequence's rows in chunks, whose partial sums are
 * rounded to fp16.  How long they are follows from max_len and the batch size
 * where all lengths need equally many chunks, else from all the lengths: the
 * low-order bits of a sequence's output may then differ with the lengths of
 * the other sequences.  A call repeats exactly for the same arguments.
 * Launch grids are sized from the host c->max_len and every length is read
 * from seq_len on the device, so a call may be captured in a graph and
 * replayed while the cache grows, provided c->max_len at capture is at least
 * every length the replays reach. */
qsvd_status qsvd_latent_decode_attention(const qsvd_layer* w, const qsvd_cache* c,
                                         const void* q, int32_t q_len, int32_t mode,
                                         float sm_scale, void* out,
                                         void* ws, size_t ws_bytes, void* stream);

/* qsvd_latent_decode_attention without a caller workspace, for callers that
 * cannot allocate device memory (code under graph capture, tight serving
 * loops, harnesses that forbid hipMalloc).  Same arguments, forms, results
 * and errors as qsvd_latent_decode_attention (and the same kernels); its
 * partial results live in a static device array of
 * qsvd_noalloc_scratch_bytes() bytes (32 MiB), one per GPU, held from the
 * first call on that GPU until the process ends.  A call whose workspace
 * query exceeds that size returns QSVD_ERR_WORKSPACE before any GPU work.
 * Calls nothing that allocates.  Every call on one GPU shares its array:
 * calls that may overlap on one GPU (other streams, other threads) race and
 * must be ordered by the caller. */
qsvd_status qsvd_latent_decode_attention_noalloc(const qsvd_layer* w, const qsvd_cache* c,
                                                 const void* q, int32_t q_len, int32_t mode,
                                                 float sm_scale, void* out, void* stream);
size_t qsvd_noalloc_scratch_bytes(void);

/* The same attention for layers that apply a rotary position embedding to q
 * and k (the paper's layers have none; this is the position-encoded variant
 * of Section 3.1's decode step).  Every rebuilt key row at position t and the
 * queries at their positions (seq_len[b] - q_len + i) are rotated before the
 * product: each head vector's pairs (j, j + head_dim/2), j < head_dim/2, are
 * turned by the angle t * rope_theta^(-2j/head_dim), formed and reduced
 * modulo one turn in fp64 and evaluated in fp32 (q_len 1: a cos/sin table
 * per call; q_len > 1: the hardware's sine and cosine of the reduced angle in
 * turns).  Values are not rotated.  Because a key then depends on
 * its position, it cannot be folded into the query, so the keys are rebuilt
 * in both forms:
 *   QSVD_ATTN_ABSORBED     K rebuilt and rotated for the scores, the value side
 *                          kept in latent space (sum_t p_t C_t, then W^u_v);
 *                          needs n_q_heads <= 32 and r in {128, 512, 1024, 1536}
 *                          (QSVD_ERR_UNSUPPORTED otherwise)
 *   QSVD_ATTN_RECONSTRUCT  K and V rebuilt, plain attention; needs
 *                          n_q_heads <= 64 and capacity <= 16384; with
 *                          q_len > 1 (query i at position seq_len[b] -
 *                          q_len + i, causal) head_dim 64 or 128
 *   QSVD_ATTN_AUTO         the first where it applies (q_len 1), else the second
 * The latent-value form takes q_len 1 (QSVD_ERR_UNSUPPORTED otherwise).  Both
 * take any cache format (F16, I8, I4), and one workspace size serves both:
 * qsvd_decode_workspace_size(w, c, q_len, QSVD_ATTN_RECONSTRUCT) bytes (the
 * same for every q_len the forms take).  rope_theta must be finite and > 1
 * (QSVD_ERR_INVALID_ARG otherwise). */
qsvd_status qsvd_latent_decode_attention_rope(const qsvd_layer* w, const qsvd_cache* c,
                                              const void* q, int32_t q_len, int32_t mode,
                                              float sm_scale, float rope_theta, void* out,
                                              void* ws, size_t ws_bytes, void* stream);

size_t qsvd_decode_workspace_size(const qsvd_layer* w, const qsvd_cache* c, int32_t q_len,
                                  int32_t mode);

/* ---- The rest of a decoder layer around the attention path ----
 * The layer's norms, its output projection and its gated MLP, on the same
 * per-token activation codes and per-channel weight codes (Section 4 setup):
 * a norm feeds qsvd_lowrank_qkv_prefill (codes), qsvd_decode_project_append
 * (fp16 rows) or a linear layer; a linear layer adds its result to the
 * residual stream that the next norm reads.  `dtype` (QSVD_F16 or QSVD_BF16)
 * is the type of every 16-bit operand of a call.  None takes a workspace. */

/* Residual addition, root-mean-square norm and per-token quantization of M rows:
 *   h  = x + residual in fp32, rounded to dtype (h = x without a residual)
 *   r  = fp32(1 / sqrt(mean_k h[k]^2 + eps)), the mean and the root in fp64
 *   y  = (h * r) * gamma in fp32, each product rounded on its own
 *   xq, sx = the quantizer of qsvd_quantize_act on the fp32 y (bits, clip)
 *   x         device [M][ldx]
 *   residual  device [M][ldr] or NULL
 *   gamma     device [K]
 *   h         device [M][ldh] or NULL (not stored); may be x or residual itself
 *             (same address and stride)
 *   y         device [M][ldy], rounded to dtype, or NULL
 *   xq        device int8 [M][K] or packed int4 [M][K/2], and sx device fp32
 *             [M], or both NULL; y or xq must be given
 * Apart from h as stated, outputs do not overlap inputs or each other.
 * A row whose a = clip * max |y| is below 2^-119 has scale 1 and codes 0, as an
 * all-zero row has (scales a / 127 then stay normal fp32 numbers, 2^-126 and
 * above; the bound is the same for 4 bits); a row with a y that is not finite (an
 * infinity or NaN in x, a sum past dtype) has scale NaN and codes 0, and other
 * rows are not affected.
 * Requires K % 8 == 0, K <= 65536, M < 2^22, strides that are multiples of 8,
 * 16-byte aligned x, residual, gamma, h and y, 8-byte aligned xq, eps > 0, bits 8
 * or 4, 0 < clip <= 1. */
qsvd_status qsvd_rmsnorm_quantize_act(const void* x, int64_t ldx, const void* residual, int64_t ldr,
                                      const void* gamma, int64_t M, int32_t K, int32_t dtype, float eps,
                                      int32_t bits, float clip, void* h, int64_t ldh, void* y, int64_t ldy,
                                      void* xq, float* sx, void* stream);

/* The gate of a gated MLP with per-token quantization of its M rows:
 *   y = gate / (1 + exp(-gate)) * up in fp32, xq, sx = the quantizer on y
 *   gate, up  device [M][ldg], [M][ldu]: the two halves of one product's rows
 *             (up = gate + K elements, ldg = ldu = 2 K) or tensors of their own
 *   xq        device int8 [M][K] or packed int4 [M][K/2]
 *   sx        device fp32 [M]
 * exp, the quotient and the product are evaluated in fp32 to a few units in the
 * last place, so a code may differ by one from that of the exact y next to a
 * rounding border; an exp(-gate) past fp32 (a gate below -88.7) makes y 0.
 * Tiny rows, values that are not finite and requirements as
 * for qsvd_rmsnorm_quantize_act. */
qsvd_status qsvd_silu_mul_quantize_act(const void* gate, int64_t ldg, const void* up, int64_t ldu, int64_t M,
                                       int32_t K, int32_t dtype, int32_t bits, float clip, void* xq, float* sx,
                                       void* stream);

/* W8A8 linear layer with a scale per token and per output channel:
 *   y[m][n] = (f32(sum_k xq[m][k] wq[n][k]) * sx[m]) * sw[n] + bias[n] + residual[m][n]
 * with an exact integer sum, every fp32 step rounded on its own (bias first,
 * then residual, each only if given) and one rounding to dtype.
 *   xq        device int8 [M][ldx], e.g. from qsvd_quantize_act with bits 8
 *   sx        device fp32 [M]
 *   wq        device int8 [N][K] (transposed: the contraction contiguous)
 *   sw        device fp32 [N]
 *   bias      device [N] or NULL
 *   residual  device [M][ldr] or NULL
 *   y         device [M][ldy]; may be residual itself (same address and stride),
 *             and overlaps no other operand
 * Requires K % 16 == 0, K < 131072, ldx % 16 == 0, ldx <= 2^22, 16-byte aligned
 * xq and wq, (M / 64 + 1) * ceil(N / 64) < 2^23; any N >= 1 and row strides of
 * residual and y (rows of y that start on 128-byte boundaries are stored fastest). */
qsvd_status qsvd_linear_i8(const void* xq, int64_t ldx, const float* sx, const void* wq, const float* sw,
                           int64_t M, int32_t N, int32_t K, const void* bias, const void* residual,
                           int64_t ldr, int32_t dtype, void* y, int64_t ldy, void* stream);

/* ---- Rotary layers: positions on several axes and a paged key/value cache ----
 * A rotary key depends on its position, so a latent cache makes every step
 * rebuild all keys; with few key/value heads a token's K and V are also no
 * wider than its latent (2 * 4 heads of 128: r = 1024).  For such layers these
 * calls turn Q and K once, keep K and V of every token in pages (16-bit rows,
 * or int8 / int4 codes with a scale per token and head), and attend over the
 * pages.  A layer's step: Q, K, V (qsvd_lowrank_qkv_prefill in fp16, or
 * qsvd_linear_i8 in either type), qsvd_rope_axes, qsvd_paged_append,
 * qsvd_paged_attention, qsvd_linear_i8.  `dtype`
 * (QSVD_F16 or QSVD_BF16) is the type of every 16-bit operand. */

enum { QSVD_ROPE_MAX_AXES = 4 };

/* How the frequencies of a rotary embedding go with the axes of a position.
 * The head_dim / 2 pairs (j, j + head_dim / 2) are dealt to the axes in runs:
 * section[0] pairs to axis 0, the next section[1] to axis 1, and so on.
 *   QSVD_ROPE_RUNNING  pair j turns by pos * theta^(-2j / head_dim), whatever its axis
 *   QSVD_ROPE_RESTART  the i-th pair of an axis with n pairs turns by pos * theta^(-i / n):
 *                      every axis has the whole range of frequencies */
enum { QSVD_ROPE_RUNNING = 0, QSVD_ROPE_RESTART = 1 };
typedef struct {
  int32_t head_dim;
  int32_t n_axes;                        /* 1 .. QSVD_ROPE_MAX_AXES */
  int32_t section[QSVD_ROPE_MAX_AXES];   /* pairs of each axis, summing to head_dim / 2 */
  int32_t order;                         /* QSVD_ROPE_RUNNING or QSVD_ROPE_RESTART */
  float   theta;                         /* finite, > 1 */
} qsvd_rope;

/* Rotary embedding of M rows of query heads and, optionally, of key heads at
 * positions with several axes: with x, y the elements j and j + head_dim / 2 of
 * a head vector and a its angle, x cos a - y sin a and y cos a + x sin a, each
 * rounded to dtype once.  The angle is formed in revolutions and reduced to
 * [0, 1) in fp64, its sine and cosine taken in fp32 (the hardware's, about
 * 2^-20 absolute).  With the same position on every axis, QSVD_ROPE_RUNNING is
 * the one-axis embedding.  Any int32 position; negated ones turn back, which is
 * also the gradient.
 *   pos     device int32 [n_axes][ldpos]: row m of axis a at pos[a * ldpos + m]
 *   q       device [M][ldq], the n_q_heads heads of a row next to each other
 *   q_out   device [M][ldqo]; may be q itself (same address and stride)
 *   k, k_out  the same for the keys, or both NULL (n_k_heads 0)
 * Requires head_dim a multiple of 16 up to 256, n_q_heads + n_k_heads <= 256,
 * M < 2^22, 16-byte aligned rows (strides that are multiples of 8). */
qsvd_status qsvd_rope_axes(const qsvd_rope* rope, const int32_t* pos, int64_t ldpos, int64_t M, int32_t dtype,
                           const void* q, int64_t ldq, int32_t n_q_heads, void* q_out, int64_t ldqo,
                           const void* k, int64_t ldk, int32_t n_k_heads, void* k_out, int64_t ldko,
                           void* stream);

/* The pages of one layer's keys and values.  A page holds page_size
 * consecutive tokens of one sequence, every head's rows together:
 *   F16   k, v are [n_pages][n_kv_heads][page_size][head_dim] of dtype, scales NULL
 *   I8    ... int8 codes, I4 packed int4 codes ([head_dim / 2] bytes), and
 *         k_scale, v_scale are fp32 [n_pages][n_kv_heads][page_size], not negative */
typedef struct {
  int32_t fmt;         /* QSVD_CACHE_*; F16 means rows of dtype */
  int32_t dtype;       /* type of K, V, Q and the outputs, and of F16 rows */
  int32_t n_kv_heads;
  int32_t head_dim;    /* 64 or 128 */
  int32_t page_size;   /* tokens: a power of two, 16 to 1024 */
  int32_t n_pages;
  void*   k;           /* device */
  void*   v;           /* device */
  float*  k_scale;     /* device or NULL (F16) */
  float*  v_scale;
} qsvd_pages;

/* What one step brings to `batch` sequences; every layer of the step uses the
 * same.  Token t of sequence b is in page page_table[b][t / page_size], row
 * t % page_size.  The step's new tokens are the last ones of each sequence:
 * rows first[b] .. first[b + 1] - 1 of Q, K, V and the outputs, at positions
 * seq_len[b] - (first[b + 1] - first[b]) .. seq_len[b] - 1.
 * A row whose position is negative, or whose page_table column is past
 * max_pages or names no page in [0, n_pages), has no place: it is not written,
 * reads as zeros, and as a key or value is not there (masked).  Rows at or
 * past first[batch] or n_rows are left alone. */
typedef struct {
  int32_t batch;
  int32_t max_pages;           /* columns of page_table */
  const int32_t* page_table;   /* device [batch][max_pages] */
  const int32_t* seq_len;      /* device [batch]: tokens after the step */
  const int32_t* first;        /* device [batch + 1], nondecreasing, first[0] = 0 */
  int32_t max_len;             /* host: at least every seq_len[b] (sizes launches) */
  int32_t max_new;             /* host: at least every first[b + 1] - first[b] */
  int64_t n_rows;              /* host: rows of Q, K, V and the outputs */
} qsvd_page_batch;

/* Write the step's new key and value rows into their pages.  I8 / I4: per row
 * and head, a = fp32(clip * max |x|) and scale = a / Qm, the code of x the
 * integer nearest to x * Qm / a within [-Qm, Qm], ties to even (the quotient is
 * formed so that one half way between two integers is met exactly); a below
 * 2^-119 gives scale 1 and codes 0, a value that is not finite gives its row and
 * head scale NaN and codes 0.  F16 rows are copied.
 *   k, v  device [n_rows][ldk], [n_rows][ldv], heads next to each other
 * Lengths and tables are not changed: the caller advances seq_len before the
 * step, once for all layers.  If two rows of a step have the same place, it is
 * left with a mixture of both (the codes of one, the scale of the other).
 * Requires n_kv_heads <= 256, n_rows and max_new < 2^22, batch <= 65536, max_len
 * <= 2^30, 16-byte aligned rows and pages, 0 < clip <= 1. */
qsvd_status qsvd_paged_append(const qsvd_pages* pages, const qsvd_page_batch* batch, const void* k, int64_t ldk,
                              const void* v, int64_t ldv, float clip, void* stream);

/* Read the rows at the step's positions back out of their pages, as dtype:
 * code * scale in fp32, rounded once.  (A batch whose new tokens are all of a
 * sequence's reads the whole sequence.)  Arguments as for qsvd_paged_append. */
qsvd_status qsvd_paged_read(const qsvd_pages* pages, const qsvd_page_batch* batch, void* k, int64_t ldk, void* v,
                            int64_t ldv, void* stream);

/* Causal attention of the step's new tokens over their sequences' pages
 * (append first, then attend): the query at position p sees the keys at
 * positions 0 .. p that are there; softmax(q k^T * sm_scale) v with fp32
 * statistics, query head h reading key/value head h / (n_q_heads /
 * n_kv_heads).  A query that sees no key gets zeros.  One token per sequence
 * (decode), chunks of a prompt, whole prompts, or all of them in one batch.
 *   q, out    device [n_rows][ldq], [n_rows][ldo], n_q_heads heads of head_dim
 *   sm_scale  0 selects 1/sqrt(head_dim)
 *   ws        device workspace of at least the size query's bytes
 * A key or value row reaches only queries that see it, also one that is NaN,
 * infinite or far larger than the others (but for low-order bits of fp16 outputs
 * over codes, where a value scale is 2^8 times larger).
 * Weights are rounded to 16 bits before they meet the values: to bf16 over bf16
 * rows, else to fp16, where a weight (over codes: times its value's scale, against
 * the largest that the query sees) loses bits below 2^-25 of the row's largest and
 * counts for nothing below 2^-36; the sum that they are divided by is off by no
 * more.  Sums are fp32: bf16 values past 2^84 may overflow them.
 * Calls that may overlap need workspaces of their own.  Lengths are read on the
 * device: a captured call may be replayed with other lengths up to max_len and
 * max_new.  A call repeats exactly for the same arguments; how a row's keys are
 * shared out, and with it the low-order bits of its outputs, follows from batch,
 * max_len, max_new and n_rows, and where sequences differ in how much they bring
 * or are long, from the lengths of the others.  A value scale past 2^125 counts
 * as infinite.
 * Requires n_q_heads a multiple of n_kv_heads and at most 256, batch <= 65536,
 * batch * n_kv_heads <= 2^18, batch * n_kv_heads * ceil(max_new * (n_q_heads /
 * n_kv_heads) / 128) <= 2^22, max_len <= 2^30, n_rows and max_new < 2^22,
 * 16-byte aligned rows, pages and ws. */
qsvd_status qsvd_paged_attention(const qsvd_pages* pages, const qsvd_page_batch* batch, const void* q, int64_t ldq,
                                 int32_t n_q_heads, float sm_scale, void* out, int64_t ldo, void* ws, size_t ws_bytes,
                                 void* stream);
size_t qsvd_paged_attention_workspace_size(const qsvd_pages* pages, const qsvd_page_batch* batch, int32_t n_q_heads);

const char* qsvd_status_string(qsvd_status s);
const char* qsvd_last_error(void);

/* Optional kernel timing.  While enabled, every kernel the library launches
 * whose name contains `filter` (all kernels if filter is NULL; the string is
 * copied) is bracketed by HIP events recorded on its launch stream;
 * qsvd_profile_read() synchronizes those events and returns the summed
 * milliseconds and launch count of the recorded kernels whose name contains
 * `name`.  Not for graph capture. */
qsvd_status qsvd_profile_enable(int32_t on, const char* filter);
qsvd_status qsvd_profile_reset(void);
qsvd_status qsvd_profile_read(const char* name, double* total_ms, int64_t* launches);

#ifdef __cplusplus
}
#endif
#endif /* QSVD_H */
