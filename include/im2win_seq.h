/*
 * im2win_seq.h -- sequence operators on AMD Instinct MI355X (gfx950).
 *
 * What follows a convolutional stem whose output pixels or frames are taken as
 * tokens: layer norm over the channels of each token, attention between the
 * tokens, and the learned bias or the rotation by which attention sees their
 * distance, each with its gradient; for serving, a key/value cache in pages,
 * also in 8 bits, and attention over it.  The same library and the same plain C
 * interface as im2win.h: host scalars and device pointers, its status codes.
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

/*
 * Rotary positions.  Of each head's D channels the first `rot` are turned in
 * pairs: channels (i, i + rot/2), or (2i, 2i+1) when interleaved, i < rot/2, by
 * the angle t = p * freq[i] of the token's position p, the others are copied:
 *   y_a = m*(x_a*cos t - x_b*sin t),  y_b = m*(x_a*sin t + x_b*cos t),  m = amplitude.
 * The backward call turns dy by -t (and multiplies by m): dx, the gradient.
 *   x, y    [B][L][H][D]: `*_stride` are the elements between sequences, tokens
 *           and heads (channels dense; not read where there is only one of
 *           them).  y may be x itself with the same strides.
 *   positions  with by_token [B][L], else [B] of the first tokens, the others
 *           following; NULL: 0, 1, ..  Any int32 values; angles are reduced in
 *           64-bit fractions of a turn, so far positions lose nothing.
 *   freq    host memory, [rot/2] radians a position, |freq| <= 1024; copied by
 *           the call.
 * rot even, 2 .. min(D, 256); D <= 2^16; H < 2^30.  Pointers need the alignment of their
 * element type only.  A lane takes up to 16 bytes of four heads; calls of 2^32
 * lanes and more are refused (IM2WIN_ERANGE).
 */
#define SEQ_ROTARY_MOST 256
typedef struct {
    int dt; /* im2win_dtype_t */
    int interleaved, by_token;
    float amplitude;
    int64_t B, L, H, D, rot;
    int64_t x_stride[3], y_stride[3];
    const int32_t *positions;
    const double *freq;
} seq_rotary_t;

int seq_rotary_forward(const seq_rotary_t *a, const void *x, void *y, void *hip_stream);
/* x_stride is dy's, y_stride dx's. */
int seq_rotary_backward(const seq_rotary_t *a, const void *dy, void *dx, void *hip_stream);

/*
 * Frequencies freq[i] = base^(-2i/rot), i < rot/2, for contexts `factor` times
 * as long as the `trained` one: a pair that turns r = trained*f/(2 pi) times
 * within the trained context keeps its frequency f from r >= high on, has
 * f/factor up to r <= low, and between them f*(w + (1-w)/factor) with
 * w = (r - low)/(high - low).  trained = 0: all pairs have f/factor (positions
 * interpolated); factor = 1: all keep f.  Host only.
 */
int seq_rotary_frequencies(double *freq, int64_t rot, double base, double factor, double trained, double low,
                           double high);

/*
 * A key/value cache in pages: a pool of `pages` pages of `page` tokens each and
 * a table that names the pages of B sequences in order.  The token at position
 * p of sequence b lies at place p % page of page table[b][p / page].  Entries
 * outside 0 .. pages-1 name no page: tokens there are neither written nor read
 * (they read as zeros and take no part in attention), nor are positions that
 * the table does not reach.
 *   k, v    [pages][page][Hkv][D] of type dt: `*_stride` are the elements
 *           between pages, tokens and heads (channels dense; not read where
 *           there is only one of them)
 *   table   [B][max_pages], rows `table_stride` entries apart (>= max_pages)
 *   k_scale, v_scale  [pages][page][Hkv] fp32, any strides, beside the codes too;
 *           8 bits only
 * dt is an im2win_dtype_t or one of 8 bits, whose numbers are codes times the
 * scale s of their token and head, with top the largest magnitude among the
 * head's D channels:
 *   SEQ_I8    s = top/127 in fp32, within 2^-126 and the largest number whose
 *             127-fold is finite, code = x/s rounded to nearest even
 *   SEQ_E4M3  s the smallest power of two >= 2^-126 with top/s <= 448, code = x/s
 *             rounded to the nearest of 4 exponent and 3 fraction bits (bias 7,
 *             no infinities)
 * A head with a value that is not finite gets the scale NaN and reads as NaN;
 * a product past the largest number of the type that is read becomes infinite.
 * D a multiple of 8, 8 .. 128; page >= 1, max_pages*page <= 2^30, pages < 2^31;
 * pages and dense operands 16-byte aligned with strides of multiples of 16
 * bytes (8-bit pages: 8 bytes); table, scales and counts as their type.
 */
enum { SEQ_I8 = 16, SEQ_E4M3 = 17 };
typedef struct {
    int dt;
    int64_t B, pages, page, max_pages, Hkv, D;
    int64_t k_stride[3], v_stride[3], k_scale_stride[3], v_scale_stride[3];
    int64_t table_stride;
    void *k, *v;
    float *k_scale, *v_scale;
    const int32_t *table;
} seq_cache_t;

/*
 * Writes new tokens: token t < count[b] of sequence b to position start[b] + t
 * (count NULL: all L; start NULL: 0).  Rows from count[b] on are not read, and
 * the pool is left as it was but for the tokens written.  The places written in one call
 * must differ (a page shared by two sequences is not written by both): where
 * two tokens meet, the place holds parts of either.
 *   k, v    [B][L][Hkv][D] of type dt (that of the cache, or any beside 8-bit
 *           pages); strides as above, of sequences, tokens and heads
 */
int seq_cache_write(const seq_cache_t *c, const void *k, const void *v, const int64_t *k_stride,
                    const int64_t *v_stride, int64_t L, im2win_dtype_t dt, const int32_t *start, const int32_t *count,
                    void *hip_stream);

/*
 * Lays sequences out densely: positions 0 .. len[b]-1 of sequence b to k and v
 * [B][L][Hkv][D]; rows from len[b] on become zeros, positions from L on are not
 * read.  Pages may be shared.
 */
int seq_cache_read(const seq_cache_t *c, void *k, void *v, const int64_t *k_stride, const int64_t *v_stride, int64_t L,
                   im2win_dtype_t dt, const int32_t *len, void *hip_stream);

/*
 * Attention of one new token of each sequence, the last of its len[b] tokens
 * (taken within 0 .. max_pages*page), over the cache: scores, out and lse as in
 * seq_attention_forward with Lq = 1, align_end and position len[b] - 1, keys
 * the tokens whose pages are there.  A sequence without any has out = 0 and
 * lse = -inf.
 *   q, out  [B][H][D] of type dt (that of the cache, or any beside 8-bit pages):
 *           `*_stride` are the elements between sequences and heads
 *   lse     [B][H] fp32
 *   ws      seq_paged_attention_workspace_bytes(c, H, dt) bytes, 16-byte aligned
 * H a multiple of Hkv, B*H < 2^24.  Scores, sums and statistics are fp32.
 * Weights over 16-bit pages are two terms of the pages' type; over 32- and 16-bit
 * pages sums of exp(s - largest) times values are divided last, and are infinite
 * past fp32's range.  8-bit codes are multiplied in fp16, which holds them exactly;
 * weights times scales are one fp16 number (two with fp32 queries) over a power of
 * two that follows the largest, so that what falls below 2^-39 of it is lost and
 * every mean of values that the type holds is reached.  bf16 and fp32 queries
 * over 8-bit pages are brought to fp16's range by a power of two a row (largest
 * channel 2^-100 or more; below, bits are lost).
 * The keys of all sequences are shared evenly between workgroups, so a sequence's
 * sums are split, and rounded, by the lengths of the others too; the same call
 * gives the same bits.
 */
typedef struct {
    int dt; /* im2win_dtype_t */
    float scale, cap;
    int64_t H;
    int64_t q_stride[2], out_stride[2];
    int64_t R;           /* range of the bias strip; 0: no bias */
    const float *strip;  /* [H][2R+1] fp32 */
    const int32_t *len;  /* [B] */
} seq_paged_attention_t;

int64_t seq_paged_attention_workspace_bytes(const seq_cache_t *c, int64_t H, im2win_dtype_t dt);
int seq_paged_attention_forward(const seq_cache_t *c, const seq_paged_attention_t *a, const void *q, void *out,
                                float *lse, void *ws, int64_t ws_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* IM2WIN_SEQ_H */
