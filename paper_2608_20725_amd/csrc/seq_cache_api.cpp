// Host side of rotary positions and the paged cache (im2win_seq.h): argument
// checks and dispatch to the kernels of seq_rotary.hip, seq_cache.hip and
// seq_paged.hip.
#include "seq_attn.hpp"
#include "seq_cache.hpp"
#include "seq_host.hpp"
#include "seq_rotary.hpp"

#include <math.h>
#include <string.h>

using namespace im2win;

namespace {

constexpr double kMaxFrequency = 1024;
constexpr int64_t kMostTokens = (int64_t)1 << 30;

// f/(2 pi) mod 1 as a fraction of 2^64, |f| <= 2^10: f's 53 bits times those of
// 2^66/(2 pi), in integers (64 pairs of long doubles took 3.6 us a call).
uint64_t turns_of(double f)
{
    constexpr uint64_t kTurn = 0xA2F9836E4E44152Au;  // 2^66/(2 pi) to the nearest
    int e;
    const uint64_t m = (uint64_t)ldexp(frexp(fabs(f), &e), 53);  // |f| = m * 2^(e-53)
    const int down = 53 - e + 2;                                 // m*kTurn >> down, 43 or more
    const uint64_t t = down < 128 ? (uint64_t)((unsigned __int128)m * kTurn >> down) : 0;
    return f < 0 ? 0 - t : t;
}

bool same_strides(const Operand &a, const Operand &b)
{
    return a.stride[0] == b.stride[0] && a.stride[1] == b.stride[1] && a.stride[2] == b.stride[2];
}

int rotary(const seq_rotary_t *a, const void *x, void *y, bool backward, void *hip_stream)
{
    if (!a || !known(a->dt) || a->B < 0 || a->L < 0 || a->H < 0 || a->D <= 0 || a->rot < 2 || a->rot % 2 ||
        a->rot > a->D || !a->freq || !isfinite(a->amplitude))
        return IM2WIN_EINVAL;
    const bool some = a->B > 0 && a->L > 0 && a->H > 0;
    if (some && (!x || !y))
        return IM2WIN_EINVAL;
    if (a->rot > SEQ_ROTARY_MOST || a->D > 1 << 16 || a->B > INT32_MAX || a->L > INT32_MAX || a->H >= 1 << 30)
        return IM2WIN_ERANGE;
    for (int64_t i = 0; i < a->rot / 2; ++i)
        if (!(fabs(a->freq[i]) <= kMaxFrequency))
            return isfinite(a->freq[i]) ? IM2WIN_ERANGE : IM2WIN_EINVAL;
    const int64_t e = elt(a->dt);
    const Operand ox(x, a->B, a->L, a->H, a->D, e, a->x_stride), oy(y, a->B, a->L, a->H, a->D, e, a->y_stride);
    int rc;
    if ((rc = check_strides(ox, true)) || (rc = check_strides(oy, true)))
        return rc;
    RotaryArgs r;
    memset(&r, 0, sizeof r);
    const bool in_place = x == y && same_strides(ox, oy);
    r.H = (int32_t)a->H, r.D = (int32_t)a->D, r.rot = (int32_t)a->rot;
    if (some && (a->B > kMaxReach / a->L || a->B * a->L > UINT32_MAX ||
                 !plan_rotary(r, a->B, a->L, a->interleaved != 0, in_place, a->dt)))
        return IM2WIN_ERANGE;
    if (!aligned(x, e) || !aligned(y, e) || !aligned(a->positions, 4))
        return IM2WIN_EALIGN;
    if (!some)
        return IM2WIN_OK;
    const Buf b[3] = {{x, ox.bytes()},
                      {y, oy.bytes()},
                      {a->positions, a->positions ? a->B * (a->by_token ? a->L : 1) * 4 : 0}};
    if ((rc = Extents().check(b, 3)))
        return rc;
    if (!self_disjoint(oy) || (!in_place && clash(ox, oy)) || meet(b[1], b[2]))
        return IM2WIN_EOVERLAP;
    if ((rc = check_device()))
        return rc;
    r.x = (const char *)x, r.y = (char *)y, r.pos = a->positions;
    r.x_sb = ox.stride[0] * e, r.x_st = ox.stride[1] * e, r.x_sh = ox.stride[2] * e;
    r.y_sb = oy.stride[0] * e, r.y_st = oy.stride[1] * e, r.y_sh = oy.stride[2] * e;
    r.by_token = a->by_token != 0;
    r.amplitude = a->amplitude, r.sin_amplitude = backward ? -a->amplitude : a->amplitude;
    Turns f;
    memset(&f, 0, sizeof f);
    for (int64_t i = 0; i < a->rot / 2; ++i)
        f.turn[i] = turns_of(a->freq[i]);
    return launch_status(launch_rotary(r, f, a->interleaved != 0, a->dt, (hipStream_t)hip_stream));
}

// ---- the cache ----

bool coded(int dt) { return dt == SEQ_I8 || dt == SEQ_E4M3; }
int64_t cache_elt(int dt) { return coded(dt) ? 1 : elt(dt); }

// The operands of a cache's description: pages stand where sequences stand in
// a dense operand, places in a page where tokens do.
struct CacheOperands {
    Operand k, v, ks, vs;
    CacheOperands(const seq_cache_t *c)
        : k(c->k, c->pages, c->page, c->Hkv, c->D, cache_elt(c->dt), c->k_stride),
          v(c->v, c->pages, c->page, c->Hkv, c->D, cache_elt(c->dt), c->v_stride),
          ks(c->k_scale, c->pages, c->page, c->Hkv, 1, 4, c->k_scale_stride),
          vs(c->v_scale, c->pages, c->page, c->Hkv, 1, 4, c->v_scale_stride)
    {
    }
};

// Dimensions, ranges and strides of a description, without its pointers.
int check_cache_dims(const seq_cache_t *c)
{
    if (!c || (!known(c->dt) && !coded(c->dt)) || c->B < 0 || c->pages < 0 || c->page <= 0 || c->max_pages < 0 ||
        c->Hkv <= 0 || c->D <= 0 || c->D % 8 || c->table_stride < c->max_pages)
        return IM2WIN_EINVAL;
    if (c->D > 128 || c->page > kMostTokens || c->max_pages > kMostTokens / c->page || c->pages > INT32_MAX ||
        c->B >= (int64_t)1 << 24 || c->Hkv >= (int64_t)1 << 24 || too_far(c->B, c->table_stride))
        return IM2WIN_ERANGE;
    const CacheOperands o(c);
    int rc;
    if ((rc = check_strides(o.k, true)) || (rc = check_strides(o.v, true)))
        return rc;
    if (coded(c->dt) && ((rc = check_strides(o.ks, true)) || (rc = check_strides(o.vs, true))))
        return rc;
    return IM2WIN_OK;
}

// Null pointers of a description whose dimensions are checked.
int check_cache_pointers(const seq_cache_t *c)
{
    if (c->pages > 0 && (!c->k || !c->v || (coded(c->dt) && (!c->k_scale || !c->v_scale))))
        return IM2WIN_EINVAL;
    if (c->B > 0 && c->max_pages > 0 && !c->table)
        return IM2WIN_EINVAL;
    return IM2WIN_OK;
}

bool strides_of(const Operand &o, int64_t bytes)
{
    return o.stride[0] * o.elt % bytes == 0 && o.stride[1] * o.elt % bytes == 0 && o.stride[2] * o.elt % bytes == 0;
}

bool cache_aligned(const seq_cache_t *c, const CacheOperands &o)
{
    const int64_t s = coded(c->dt) ? 8 : 16;
    return aligned(c->k, 16) && aligned(c->v, 16) && strides_of(o.k, s) && strides_of(o.v, s) &&
           aligned(c->table, 4) && (!coded(c->dt) || (aligned(c->k_scale, 4) && aligned(c->v_scale, 4)));
}

Buf buf_of(const Operand &o) { return Buf{o.p, o.bytes()}; }

// The cache's buffers; `most` of them.
constexpr int kCacheBufs = 5;
void cache_bufs(const seq_cache_t *c, const CacheOperands &o, Buf *b)
{
    const bool any = c->B > 0 && c->max_pages > 0;
    b[0] = buf_of(o.k), b[1] = buf_of(o.v);
    b[2] = Buf{c->table, any ? ((c->B - 1) * c->table_stride + c->max_pages) * 4 : 0};
    b[3] = b[4] = Buf{nullptr, 0};
    if (coded(c->dt))
        b[3] = buf_of(o.ks), b[4] = buf_of(o.vs);
}

Pool make_pool(const seq_cache_t *c, const CacheOperands &o)
{
    Pool p;
    memset(&p, 0, sizeof p);
    p.k = (char *)c->k, p.v = (char *)c->v;
    const auto set = [](const Operand &s, int64_t &page, int64_t &tok, int64_t &head) {
        page = s.stride[0] * s.elt, tok = s.stride[1] * s.elt, head = s.stride[2] * s.elt;
    };
    set(o.k, p.k_page, p.k_tok, p.k_head);
    set(o.v, p.v_page, p.v_tok, p.v_head);
    if (coded(c->dt)) {
        p.ks = (char *)c->k_scale, p.vs = (char *)c->v_scale;
        set(o.ks, p.ks_page, p.ks_tok, p.ks_head);
        set(o.vs, p.vs_page, p.vs_tok, p.vs_head);
    }
    p.table = c->table, p.table_stride = c->table_stride;
    p.page = make_fastdiv((uint32_t)c->page);
    p.pages = (int32_t)c->pages, p.max_pages = (int32_t)c->max_pages;
    p.Hkv = (int32_t)c->Hkv, p.D = (int32_t)c->D;
    return p;
}

int copy(const seq_cache_t *c, const void *k, const void *v, const int64_t *k_stride, const int64_t *v_stride,
         int64_t L, int dt, const int32_t *start, const int32_t *count, void *hip_stream, bool write)
{
    int rc;
    if ((rc = check_cache_dims(c)))
        return rc;
    if (!known(dt) || (!coded(c->dt) && dt != c->dt) || L < 0 || !k_stride || !v_stride)
        return IM2WIN_EINVAL;
    const bool some = c->B > 0 && L > 0;
    if ((rc = check_cache_pointers(c)) || (some && (!k || !v || (!write && !count))))
        return rc ? rc : IM2WIN_EINVAL;
    if (L > kMostTokens || (some && (c->B > kMaxReach / L || c->B * L > kMaxReach / c->Hkv ||
                                     !cache_grid_fits(c->B, L, c->Hkv, c->D))))
        return IM2WIN_ERANGE;
    const int64_t e = elt(dt);
    const Operand ok(k, c->B, L, c->Hkv, c->D, e, k_stride), ov(v, c->B, L, c->Hkv, c->D, e, v_stride);
    if ((rc = check_strides(ok, true)) || (rc = check_strides(ov, true)))
        return rc;
    const CacheOperands o(c);
    if (!cache_aligned(c, o) || !aligned(k, 16) || !aligned(v, 16) || !strides_of(ok, 16) || !strides_of(ov, 16) ||
        !aligned(start, 4) || !aligned(count, 4))
        return IM2WIN_EALIGN;
    if (!some)
        return IM2WIN_OK;
    Buf own[kCacheBufs];
    cache_bufs(c, o, own);
    const Buf dense[4] = {buf_of(ok), buf_of(ov), {start, start ? c->B * 4 : 0}, {count, count ? c->B * 4 : 0}};
    Extents ext;
    if ((rc = ext.check(own, kCacheBufs)) || (rc = ext.check(dense, 4)))
        return rc;
    if (write) {
        if (!self_disjoint(o.k) || !self_disjoint(o.v) || clash(o.k, o.v))
            return IM2WIN_EOVERLAP;
        // scales may lie beside the codes, in the same pages
        if (coded(c->dt) && (!self_disjoint(o.ks) || !self_disjoint(o.vs) || clash(o.ks, o.vs) || clash(o.k, o.ks) ||
                             clash(o.k, o.vs) || clash(o.v, o.ks) || clash(o.v, o.vs)))
            return IM2WIN_EOVERLAP;
        const int outs[4] = {0, 1, 3, 4};
        for (const int i : outs) {
            if (meet(own[i], own[2]))
                return IM2WIN_EOVERLAP;
            for (const Buf &d : dense)
                if (meet(own[i], d))
                    return IM2WIN_EOVERLAP;
        }
    } else {
        if (!self_disjoint(ok) || !self_disjoint(ov) || clash(ok, ov))
            return IM2WIN_EOVERLAP;
        for (int i = 0; i < 2; ++i) {
            for (const Buf &b : own)
                if (meet(dense[i], b))
                    return IM2WIN_EOVERLAP;
            if (meet(dense[i], dense[3]))
                return IM2WIN_EOVERLAP;
        }
    }
    if ((rc = check_device()))
        return rc;
    Dense d;
    memset(&d, 0, sizeof d);
    d.k = (char *)k, d.v = (char *)v;
    d.k_sb = ok.stride[0] * e, d.k_st = ok.stride[1] * e, d.k_sh = ok.stride[2] * e;
    d.v_sb = ov.stride[0] * e, d.v_st = ov.stride[1] * e, d.v_sh = ov.stride[2] * e;
    d.start = start, d.count = count;
    d.B = (int32_t)c->B, d.L = (int32_t)L;
    d.len = make_fastdiv((uint32_t)L), d.heads = make_fastdiv((uint32_t)c->Hkv);
    const Pool p = make_pool(c, o);
    const hipStream_t st = (hipStream_t)hip_stream;
    return launch_status(write ? launch_cache_write(p, c->dt, d, dt, st) : launch_cache_read(p, c->dt, d, dt, st));
}

int check_heads(const seq_cache_t *c, int64_t H, int dt)
{
    if (!known(dt) || (!coded(c->dt) && dt != c->dt) || H <= 0 || H % c->Hkv)
        return IM2WIN_EINVAL;
    if (H >= (int64_t)1 << 24 || c->B * H >= (int64_t)1 << 24)
        return IM2WIN_ERANGE;
    return IM2WIN_OK;
}

}  // namespace

extern "C" {

int seq_rotary_forward(const seq_rotary_t *a, const void *x, void *y, void *hip_stream)
{
    return rotary(a, x, y, false, hip_stream);
}

int seq_rotary_backward(const seq_rotary_t *a, const void *dy, void *dx, void *hip_stream)
{
    return rotary(a, dy, dx, true, hip_stream);
}

int seq_rotary_frequencies(double *freq, int64_t rot, double base, double factor, double trained, double low,
                           double high)
{
    if (!freq || rot < 2 || rot % 2 || !(base >= 1) || !isfinite(base) || !(factor >= 1) || !isfinite(factor) ||
        !(trained >= 0) || !isfinite(trained) || !isfinite(low) || !isfinite(high) || (trained > 0 && !(high > low)))
        return IM2WIN_EINVAL;
    if (rot > SEQ_ROTARY_MOST)
        return IM2WIN_ERANGE;
    for (int64_t i = 0; i < rot / 2; ++i) {
        const double f = pow(base, -2.0 * (double)i / (double)rot);
        double w = 0;
        if (trained > 0) {
            w = (trained * f / (2 * M_PI) - low) / (high - low);
            w = w < 0 ? 0 : w > 1 ? 1 : w;
        }
        freq[i] = f * w + f / factor * (1 - w);
    }
    return IM2WIN_OK;
}

int seq_cache_write(const seq_cache_t *c, const void *k, const void *v, const int64_t *k_stride,
                    const int64_t *v_stride, int64_t L, im2win_dtype_t dt, const int32_t *start, const int32_t *count,
                    void *hip_stream)
{
    return copy(c, k, v, k_stride, v_stride, L, dt, start, count, hip_stream, true);
}

int seq_cache_read(const seq_cache_t *c, void *k, void *v, const int64_t *k_stride, const int64_t *v_stride, int64_t L,
                   im2win_dtype_t dt, const int32_t *len, void *hip_stream)
{
    return copy(c, k, v, k_stride, v_stride, L, dt, nullptr, len, hip_stream, false);
}

int64_t seq_paged_attention_workspace_bytes(const seq_cache_t *c, int64_t H, im2win_dtype_t dt)
{
    int rc;
    if ((rc = check_cache_dims(c)) || (rc = check_heads(c, H, dt)))
        return rc;
    return pad256(paged_part_floats(make_pool(c, CacheOperands(c)), c->dt, c->B, H, dt) * 4);
}

int seq_paged_attention_forward(const seq_cache_t *c, const seq_paged_attention_t *a, const void *q, void *out,
                                float *lse, void *ws, int64_t ws_bytes, void *hip_stream)
{
    int rc;
    if ((rc = check_cache_dims(c)))
        return rc;
    if (!a)
        return IM2WIN_EINVAL;
    if ((rc = check_heads(c, a->H, a->dt)))
        return rc;
    if (!isfinite(a->scale) || !isfinite(a->cap) || a->cap < 0 || a->R < 0)
        return IM2WIN_EINVAL;
    if ((rc = check_cache_pointers(c)) || (c->B > 0 && (!q || !out || !lse || !a->len)) || (a->R && !a->strip))
        return rc ? rc : IM2WIN_EINVAL;
    if (a->R > SEQ_BIAS_RANGE)
        return IM2WIN_ERANGE;
    // one token a sequence: its stride is never read
    const int64_t e = elt(a->dt);
    const int64_t qs[3] = {a->q_stride[0], 0, a->q_stride[1]}, os[3] = {a->out_stride[0], 0, a->out_stride[1]};
    const Operand oq(q, c->B, 1, a->H, c->D, e, qs), oo(out, c->B, 1, a->H, c->D, e, os);
    if ((rc = check_strides(oq)) || (rc = check_strides(oo)))
        return rc;
    const CacheOperands o(c);
    if (!cache_aligned(c, o) || !aligned(q, 16) || !aligned(out, 16) || !strides_of(oq, 16) || !strides_of(oo, 16) ||
        !aligned(lse, 4) || !aligned(a->len, 4) || !aligned(a->strip, 4) || !aligned(ws, 16))
        return IM2WIN_EALIGN;
    if (ws_bytes < 0)
        return IM2WIN_EWORKSPACE;
    if (c->B == 0)
        return IM2WIN_OK;
    Buf own[kCacheBufs];
    cache_bufs(c, o, own);
    const Buf in[3] = {buf_of(oq), {a->len, c->B * 4}, {a->strip, a->R ? a->H * (2 * a->R + 1) * 4 : 0}};
    const Buf outs[3] = {buf_of(oo), {lse, c->B * a->H * 4}, {ws, ws ? ws_bytes : 0}};
    Extents ext;
    if ((rc = ext.check(own, kCacheBufs)) || (rc = ext.check(in, 3)) || (rc = ext.check(outs, 3)))
        return rc;
    if (!self_disjoint(oo) || clash(oo, oq))
        return IM2WIN_EOVERLAP;
    for (int i = 0; i < 3; ++i) {
        for (const Buf &b : own)
            if (meet(outs[i], b))
                return IM2WIN_EOVERLAP;
        for (int j = 0; j < 3; ++j)
            if (!(i == 0 && j == 0) && meet(outs[i], in[j]))  // out and q may be columns of one tensor
                return IM2WIN_EOVERLAP;
        for (int j = 0; j < i; ++j)
            if (meet(outs[i], outs[j]))
                return IM2WIN_EOVERLAP;
    }
    const Pool p = make_pool(c, o);
    const int64_t need = pad256(paged_part_floats(p, c->dt, c->B, a->H, a->dt) * 4);
    if (need > 0 && (!ws || ws_bytes < need))
        return IM2WIN_EWORKSPACE;
    if ((rc = check_device()))
        return rc;
    PagedArgs r;
    memset(&r, 0, sizeof r);
    r.q = (const char *)q, r.out = (char *)out, r.lse = lse, r.part = (float *)ws;
    r.len = a->len, r.strip = a->strip;
    r.q_sb = oq.stride[0] * e, r.q_sh = oq.stride[2] * e, r.o_sb = oo.stride[0] * e, r.o_sh = oo.stride[2] * e;
    r.B = (int32_t)c->B, r.H = (int32_t)a->H, r.G = (int32_t)(a->H / c->Hkv), r.R = (int32_t)a->R;
    r.scale = a->scale, r.cap = a->cap;
    return launch_status(launch_paged(p, c->dt, r, a->dt, (hipStream_t)hip_stream));
}

}  // extern "C"
