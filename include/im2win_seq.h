/*
 * im2win_seq.h -- sequence operators on AMD Instinct MI355X (gfx950).
 *
 * What follows a convolutional stem whose output pixels or frames are taken as
 * tokens: layer norm over the channels of each token, attention between the
 * tokens, and the learned bias by which attention sees their distance, each
 * with its gradient.  The same library and the same plain C interface as
 * im2win.h: host scalars and device pointers, status codes of im2win.h.
 *
 * Ownership: the caller allocates every buffer; the library allocates nothing.
 * Streams: every device call only enqueues work on `hip_stream` (a
 * hipStream_t; NULL is the null stream) and returns without synchronising; it
 * can be captured into a HIP graph.  Buffers, workspaces among them, belong to
 * the call until that work has ended.
 * Results do not depend on launch order: every sum is taken in a fixed order
 * (the atomics on LDS in the bias strip's gradient have an address a lane each
 * and one wave that adds), so the same call on the same inputs gives the same
 * bits.
 * Numerics: sums, means, softmax statistics and gradients are held in fp32;
 * fp16 and bf16 results are rounded once, to nearest even, on store.  The
 * 16-bit attention kernels also round the softmax weights P and, in the
 * backward pass, the score gradients to the element type, as operands of the
 * matrix cores.
 * Errors: arguments are checked before anything is enqueued, in this order:
 * null pointers and dimensions -> index ranges -> alignment -> buffer extents
 * -> overlap -> workspace size -> device -> launch.  The first failing check's
 * status is returned.  Counts of zero rows, sequences, queries or keys are
 * valid; the pointers of buffers without elements may be NULL.
 */
#ifndef IM2WIN_SEQ_H
#define IM2WIN_SEQ_H

#include "im2win.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Layer norm of each row x[r][0 .. C):
 *   mean = sum(x)/C,  rstd = (sum((x - mean)^2)/C + eps)^(-1/2),
 *   y = (x - mean)*rstd*weight + bias.
 *   x       [rows][C], rows `x_stride` elements apart (>= C; channels dense)
 *   weight, bias  [C] of type `wdt`: dt, or IM2WIN_F32 beside 16-bit rows
 *   y       [rows][C] dense, type dt; may be x itself when x_stride == C
 *   mean, rstd    [rows] fp32 (for the backward call)
 * Pointers need the alignment of their element type only.  C < 2^24,
 * rows < 2^31.
 */
int seq_layer_norm_forward(const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd,
                           int64_t rows, int64_t C, int64_t x_stride, float eps, im2win_dtype_t dt,
                           im2win_dtype_t wdt, void *hip_stream);

/*
 * Its gradients, with xh = (x - mean)*rstd and g = dy*weight:
 *   dx = rstd*(g - mean(g) - xh*mean(g*xh)) [rows][C] dense, type dt,
 *   dweight = sum over rows of dy*xh, dbias = sum over rows of dy, [C], type wdt.
 *   dy      [rows][C], rows `dy_stride` elements apart
 *   ws      seq_layer_norm_workspace_bytes(rows, C) bytes, 16-byte aligned
 */
int64_t seq_layer_norm_workspace_bytes(int64_t rows, int64_t C);
int seq_layer_norm_backward(const void *dy, const void *x, const void *weight, const float *mean, const float *rstd,
                            void *dx, void *dweight, void *dbias, void *ws, int64_t ws_bytes, int64_t rows, int64_t C,
                            int64_t dy_stride, int64_t x_stride, im2win_dtype_t dt, im2win_dtype_t wdt,
                            void *hip_stream);

/*
 * Learned bias by buckets of the distance d = key position - query position.
 * Buckets 0 .. m-1 hold n = |d| when two_sided (m = buckets/2; the keys after
 * the query, d > 0, take buckets m .. 2m-1) or n = max(-d, 0) (m = buckets),
 * with e = floor(m/2):
 *   n < e: bucket n;  else min(m-1, floor(e + (m-e)*ln(n/e)/ln(R/e) + 1e-9)).
 * From |d| = R on the bucket no longer changes, so a strip of 2R+1 values per
 * head holds the bias of every distance.
 *   table   [buckets][H], type dt
 *   strip   [H][2R+1] fp32: strip[h][d + R] = table[bucket(d)][h]
 * 2 <= m <= 512, buckets even when two_sided, e < R <= SEQ_BIAS_RANGE, H < 2^16.
 */
#define SEQ_BIAS_RANGE 1024
int seq_rel_bias_forward(const void *table, float *strip, int64_t H, int64_t buckets, int64_t R, int two_sided,
                         im2win_dtype_t dt, void *hip_stream);

/*
 * dtable[b][h] = sum over n and over the distances d of bucket b of
 * dstrip[n][h][d + R] (n: the attention layers that share the table).
 */
int seq_rel_bias_backward(const float *dstrip, void *dtable, int64_t n, int64_t H, int64_t buckets, int64_t R,
                          int two_sided, im2win_dtype_t dt, void *hip_stream);

/*
 * The bucket of distance d (clamped to -R .. R).  Host only.  Returns the
 * bucket, or IM2WIN_EINVAL / IM2WIN_ERANGE.
 */
int64_t seq_rel_bias_bucket(int64_t d, int64_t buckets, int64_t R, int two_sided);

/*
 * Attention.  Query i of a sequence with n keys (kv_len, else Lk) is at
 * position p = i, or with align_end p = i + n - Lq; key j is at position j.
 *   score  s = c(scale * q.k) + strip[h][clamp(j - p, -R, R) + R],
 *          c(x) = cap*tanh(x/cap), or x when cap is 0
 * over the pairs that take part: j < n; when causal, j <= p or j < prefix;
 * with documents, q_doc[i] == k_doc[j] >= 0.  Then
 *   lse = ln(sum exp(s)),  P = exp(s - lse),  out = sum P*v.
 * A query without pairs has out = 0, lse = -inf and no part in any gradient.
 * Left-out pairs have no influence, whatever their keys and values hold.
 *
 * q [B][Lq][H][D], k and v [B][Lk][Hkv][D], out like q: `*_stride` are the
 * elements between sequences, tokens and heads (channels dense; not read where
 * there is only one of them).  Head h reads
 * key/value head h / (H / Hkv).  lse [B][H][Lq] dense fp32.
 * D a multiple of 8, 8 .. 128; H a multiple of Hkv; Lq, Lk <= 2^20;
 * B*H*max(1, ceil(Lq/128)) < 2^24 (backward B*H*ceil(Lq/64) +
 * B*Hkv*ceil(Lk/64) < 2^24), with documents B*ceil(Lq/64) and B*ceil(Lk/64)
 * < 2^26; strides multiples of 16 bytes, token strides below 2^24 bytes;
 * pointers of 16-bit and fp32 rows 16-byte aligned.
 */
typedef struct {
    int dt; /* im2win_dtype_t */
    int causal, align_end;
    float scale, cap;
    int64_t B, Lq, Lk, H, Hkv, D;
    int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3];
    int64_t dout_stride[3], dq_stride[3], dk_stride[3], dv_stride[3]; /* backward call only */
    int64_t R;             /* range of the bias strip; 0: no bias */
    const float *strip;    /* [H][2R+1] fp32 */
    const int32_t *kv_len; /* [B], or NULL; values are taken within 0 .. Lk */
    const int32_t *prefix; /* [B], or NULL; read when causal */
    const int32_t *q_doc;  /* [B][Lq], with k_doc, or NULL */
    const int32_t *k_doc;  /* [B][Lk] */
} seq_attention_t;

/* Workspace of the forward (backward = 0) or backward call (16-byte aligned); 0 when none is needed. */
int64_t seq_attention_workspace_bytes(const seq_attention_t *a, int backward);

int seq_attention_forward(const seq_attention_t *a, const void *q, const void *k, const void *v, void *out, float *lse,
                          void *ws, int64_t ws_bytes, void *hip_stream);

/*
 * Gradients from dout (like q) and the forward call's out and lse, with
 * dS = P*(dout.v - dout.out): dv = sum P*dout, dq and dk through
 * scale*(1 - (c/cap)^2)*dS, and dstrip[h][d + R] = sum of dS over the pairs of
 * that (clamped) distance in all sequences.  Shared key/value heads receive
 * the sum over their query heads.
 *   dstrip  [H][2R+1] fp32; NULL when R is 0 (or when its gradient is not wanted)
 */
int seq_attention_backward(const seq_attention_t *a, const void *dout, const void *q, const void *k, const void *v,
                           const void *out, const float *lse, void *dq, void *dk, void *dv, float *dstrip, void *ws,
                           int64_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* IM2WIN_SEQ_H */
