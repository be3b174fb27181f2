// Host side of the sequence operators (im2win_seq.h): argument checks,
// workspace accounting and dispatch to the kernels of seq_norm.hip,
// seq_bias.hip and seq_attn_*.hip.
#include "seq_attn.hpp"

#include <math.h>
#include <string.h>

using namespace im2win;

namespace {

constexpr int64_t kMaxLen = int64_t(1) << 20;
constexpr int64_t kMaxReach = int64_t(1) << 44;  // elements between the first and the last of an axis: no memory is larger

bool too_far(int64_t n, int64_t stride) { return n > 1 && stride > kMaxReach / (n - 1); }
bool known(int dt) { return dt == IM2WIN_F32 || dt == IM2WIN_F16 || dt == IM2WIN_BF16; }
int64_t elt(int dt) { return dt == IM2WIN_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t a) { return ((uintptr_t)p & (uintptr_t)(a - 1)) == 0; }
int64_t pad256(int64_t n) { return (n + 255) / 256 * 256; }

// A buffer of a call: the bytes from p on that it may touch.
struct Buf {
    const void *p;
    int64_t bytes;
};

// Checks that buffers lie in one device allocation each.  The allocations that
// a call has met are kept for its other buffers: asking the runtime takes 0.2
// us a buffer, and an allocator serves many tensors from one allocation.
class Extents {
public:
    int check(const Buf *b, int n)
    {
        for (int i = 0; i < n; ++i)
            if (b[i].bytes > 0)
                if (const int rc = one(b[i]))
                    return rc;
        return IM2WIN_OK;
    }

private:
    static constexpr int kMost = 8;
    uintptr_t base_[kMost];
    uint64_t size_[kMost];
    int n_ = 0;

    static bool inside(const Buf &b, uintptr_t base, uint64_t size)
    {
        const uintptr_t q = (uintptr_t)b.p;
        return q >= base && (uint64_t)(q - base) + (uint64_t)b.bytes <= size;
    }
    int one(const Buf &b)
    {
        for (int i = 0; i < n_; ++i)
            if (inside(b, base_[i], size_[i]))
                return IM2WIN_OK;
        hipDeviceptr_t base = nullptr;
        size_t size = 0;
        if (hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)b.p) != hipSuccess) {
            (void)hipGetLastError();  // leave no sticky error behind for the caller
            return IM2WIN_EBUFFER;
        }
        if (!inside(b, (uintptr_t)base, size))
            return IM2WIN_EBUFFER;
        if (n_ < kMost) {
            base_[n_] = (uintptr_t)base;
            size_[n_++] = size;
        }
        return IM2WIN_OK;
    }
};

bool meet(const Buf &a, const Buf &b) { return a.bytes > 0 && b.bytes > 0 && overlaps(a.p, a.bytes, b.p, b.bytes); }

// ---- attention ----

// One operand [B][L][heads][D] in memory.
struct Operand {
    const void *p;
    int64_t B, L, heads, D, elt;
    int64_t stride[3];  // elements: sequence, token, head; 0 where there is one of them (or none): nothing steps

    Operand(const void *ptr, int64_t b, int64_t l, int64_t h, int64_t d, int64_t e, const int64_t *s)
        : p(ptr), B(b), L(l), heads(h), D(d), elt(e), stride{b > 1 ? s[0] : 0, l > 1 ? s[1] : 0, h > 1 ? s[2] : 0}
    {
    }
    int64_t bytes() const  // from the first element to the end of the last
    {
        if (B == 0 || L == 0)
            return 0;
        return ((B - 1) * stride[0] + (L - 1) * stride[1] + (heads - 1) * stride[2] + D) * elt;
    }
};

int check_strides(const Operand &o)
{
    const int64_t n[3] = {o.B, o.L, o.heads};
    for (int k = 0; k < 3; ++k) {
        if (o.stride[k] < 0)
            return IM2WIN_EINVAL;
        if (too_far(n[k], o.stride[k]))
            return IM2WIN_ERANGE;
    }
    if (o.stride[1] * o.elt >= (int64_t)1 << 24)
        return IM2WIN_ERANGE;
    return IM2WIN_OK;
}

// Rows of an output must not meet each other: heads within a token, tokens
// within a sequence (or the other way round), sequences apart.
bool self_disjoint(const Operand &o)
{
    struct Axis {
        int64_t n, s;
    } ax[3] = {{o.B, o.stride[0]}, {o.L, o.stride[1]}, {o.heads, o.stride[2]}};
    for (int i = 0; i < 2; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (ax[j].s < ax[i].s) {
                const Axis t = ax[i];
                ax[i] = ax[j];
                ax[j] = t;
            }
    int64_t reach = o.D;  // elements one step of the next axis has to clear
    for (int i = 0; i < 3; ++i) {
        if (ax[i].n > 1 && ax[i].s < reach)
            return false;
        reach += (ax[i].n - 1) * ax[i].s;
    }
    return true;
}

// Bytes modulo `period` that an operand takes from its first element on: the
// axes that step by whole periods add none.
int64_t width(const Operand &o, int64_t period)
{
    const int64_t n[3] = {o.B, o.L, o.heads};
    int64_t w = o.D;
    for (int k = 0; k < 3; ++k)
        if (n[k] > 1 && o.stride[k] % period)
            w += (n[k] - 1) * o.stride[k];
    return w * o.elt;
}

// Two operands whose extents meet may still lie side by side, as q, k and v do
// in one tensor: there is a stride (the tokens', if they are columns of each
// token's row; the sequences' or heads' in other orders of the dimensions)
// modulo which their bytes are apart.
bool side_by_side(const Operand &a, const Operand &b)
{
    const int64_t n[6] = {a.B, a.L, a.heads, b.B, b.L, b.heads};
    const int64_t diff = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
    for (int k = 0; k < 6; ++k) {
        const int64_t period = k < 3 ? a.stride[k] : b.stride[k - 3], bytes = period * a.elt;
        if (n[k] <= 1 || period <= 0)
            continue;
        const int64_t off = ((diff % bytes) + bytes) % bytes;  // where b starts, a's start being 0
        if (off >= width(a, period) && off + width(b, period) <= bytes)
            return true;
    }
    return false;
}

bool clash(const Operand &a, const Operand &b)
{
    const Buf x{a.p, a.bytes()}, y{b.p, b.bytes()};
    return meet(x, y) && !side_by_side(a, b);
}

struct Sizes {
    int64_t stat, norms, q_range, k_range, part, total;
};

// Dimensions and ranges of a description, without its pointers.
int check_dims(const seq_attention_t *a, bool backward)
{
    if (!a || !known(a->dt))
        return IM2WIN_EINVAL;
    if (a->B < 0 || a->Lq < 0 || a->Lk < 0 || a->H <= 0 || a->Hkv <= 0 || a->D <= 0 || a->R < 0 || a->H % a->Hkv)
        return IM2WIN_EINVAL;
    if (a->D % 8 || !isfinite(a->scale) || !isfinite(a->cap) || a->cap < 0)
        return IM2WIN_EINVAL;
    if (a->D > 128 || a->Lq > kMaxLen || a->Lk > kMaxLen || a->R > SEQ_BIAS_RANGE)
        return IM2WIN_ERANGE;
    if (a->H >= (int64_t)1 << 24 || a->B >= (int64_t)1 << 24 || a->B * a->H >= (int64_t)1 << 24)
        return IM2WIN_ERANGE;
    // A grid has less than 2^32 lanes: 2^24 workgroups of 256.  (The launches
    // with splits and the joins are small ones, and few rows make at most
    // B*H workgroups.)
    constexpr int64_t most = (int64_t)1 << 24;
    const int64_t heads = a->B * a->H, longest = a->Lq > a->Lk ? a->Lq : a->Lk;
    if (!backward && heads * ((a->Lq + kHeld - 1) / kHeld) >= most)
        return IM2WIN_ERANGE;
    if (backward && heads * ((a->Lq + 63) / 64) + a->B * a->Hkv * ((a->Lk + 63) / 64) >= most)
        return IM2WIN_ERANGE;
    if ((a->q_doc || a->k_doc) && a->B * ((longest + kDocTile - 1) / kDocTile) >= most * 4)  // one wave each
        return IM2WIN_ERANGE;
    const int64_t e = elt(a->dt);
    const Operand ops[4] = {{nullptr, a->B, a->Lq, a->H, a->D, e, a->q_stride},
                            {nullptr, a->B, a->Lk, a->Hkv, a->D, e, a->k_stride},
                            {nullptr, a->B, a->Lk, a->Hkv, a->D, e, a->v_stride},
                            {nullptr, a->B, a->Lq, a->H, a->D, e, a->out_stride}};
    for (const Operand &o : ops)
        if (const int rc = check_strides(o))
            return rc;
    if (!self_disjoint(ops[3]))
        return IM2WIN_EOVERLAP;
    if (!backward)
        return IM2WIN_OK;
    const Operand back[4] = {{nullptr, a->B, a->Lq, a->H, a->D, e, a->dout_stride},
                             {nullptr, a->B, a->Lq, a->H, a->D, e, a->dq_stride},
                             {nullptr, a->B, a->Lk, a->Hkv, a->D, e, a->dk_stride},
                             {nullptr, a->B, a->Lk, a->Hkv, a->D, e, a->dv_stride}};
    for (const Operand &o : back)
        if (const int rc = check_strides(o))
            return rc;
    for (int k = 1; k < 4; ++k)
        if (!self_disjoint(back[k]))
            return IM2WIN_EOVERLAP;
    return IM2WIN_OK;
}

bool strides_aligned(const int64_t *s, int64_t B, int64_t L, int64_t heads, int64_t e)
{
    return (B <= 1 || s[0] * e % 16 == 0) && (L <= 1 || s[1] * e % 16 == 0) && (heads <= 1 || s[2] * e % 16 == 0);
}

Sizes sizes_of(const seq_attention_t *a, bool backward)
{
    Sizes s;
    memset(&s, 0, sizeof s);
    if (a->q_doc || a->k_doc) {
        s.q_range = pad256(a->B * ((a->Lq + kDocTile - 1) / kDocTile) * (int64_t)sizeof(DocRange));
        s.k_range = pad256(a->B * ((a->Lk + kDocTile - 1) / kDocTile) * (int64_t)sizeof(DocRange));
    }
    if (backward) {
        s.stat = pad256(a->B * a->H * ((a->Lq + 63) / 64 * 64) * 8);
        s.norms = a->dt == IM2WIN_F16 ? pad256(attn_norm_bytes(a->B, a->Lq, a->Lk, a->H, a->Hkv)) : 0;
    }
    s.part = pad256(attn_part_bytes(a->dt, a->B, a->Lq, a->Lk, a->H, a->Hkv, a->D, a->R, backward));
    s.total = s.stat + s.norms + s.q_range + s.k_range + s.part;
    return s;
}

// An operand's strides in bytes.
void set_strides(const Operand &o, int64_t &sequence, int32_t &token, int64_t &head)
{
    sequence = o.stride[0] * o.elt;
    token = (int32_t)(o.stride[1] * o.elt);
    head = o.stride[2] * o.elt;
}

AttnArgs make_args(const seq_attention_t *a)
{
    AttnArgs r;
    memset(&r, 0, sizeof r);
    const int64_t e = elt(a->dt);
    const Operand q(nullptr, a->B, a->Lq, a->H, a->D, e, a->q_stride), k(nullptr, a->B, a->Lk, a->Hkv, a->D, e, a->k_stride),
        v(nullptr, a->B, a->Lk, a->Hkv, a->D, e, a->v_stride), o(nullptr, a->B, a->Lq, a->H, a->D, e, a->out_stride);
    set_strides(q, r.q_sb, r.q_st, r.q_sh);
    set_strides(k, r.k_sb, r.k_st, r.k_sh);
    set_strides(v, r.v_sb, r.v_st, r.v_sh);
    set_strides(o, r.o_sb, r.o_st, r.o_sh);
    r.B = (int32_t)a->B, r.Lq = (int32_t)a->Lq, r.Lk = (int32_t)a->Lk;
    r.H = (int32_t)a->H, r.Hkv = (int32_t)a->Hkv, r.G = (int32_t)(a->H / a->Hkv), r.D = (int32_t)a->D;
    r.causal = a->causal != 0, r.align_end = a->align_end != 0;
    r.scale = a->scale, r.cap = a->cap;
    if (a->R) {
        r.R = (int32_t)attn_range(a->R, a->Lq, a->Lk), r.strip_step = 2 * a->R + 1;
        r.strip = a->strip + (a->R - r.R);
    }
    r.kv_len = a->kv_len, r.prefix = a->causal ? a->prefix : nullptr;
    r.q_doc = a->q_doc, r.k_doc = a->k_doc;
    return r;
}

// Places the workspace's parts and fills the documents' ranges.
int place(AttnArgs *r, const seq_attention_t *a, const Sizes &s, void *ws, hipStream_t st)
{
    char *p = (char *)ws;
    r->stat = (float *)p, p += s.stat;
    r->norms = (float *)p, p += s.norms;
    DocRange *qr = (DocRange *)p;
    p += s.q_range;
    DocRange *kr = (DocRange *)p;
    p += s.k_range;
    r->part = (float *)p;
    if (!a->q_doc)
        return IM2WIN_OK;
    r->q_range = qr, r->k_range = kr;
    int rc;
    if ((rc = launch_status(launch_attn_docs(a->q_doc, qr, a->B, a->Lq, st))))
        return rc;
    return launch_status(launch_attn_docs(a->k_doc, kr, a->B, a->Lk, st));
}

}  // namespace

extern "C" {

int seq_layer_norm_forward(const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd,
                           int64_t rows, int64_t C, int64_t x_stride, float eps, im2win_dtype_t dt, im2win_dtype_t wdt,
                           void *hip_stream)
{
    if (!known(dt) || (wdt != dt && wdt != IM2WIN_F32) || rows < 0 || C <= 0 || x_stride < C || !(eps >= 0))
        return IM2WIN_EINVAL;
    if (!weight || !bias || (rows > 0 && (!x || !y || !mean || !rstd)))
        return IM2WIN_EINVAL;
    if (rows > INT32_MAX || C >= (int64_t)1 << 24 || too_far(rows, x_stride))
        return IM2WIN_ERANGE;
    const int64_t e = elt(dt), we = elt(wdt);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(weight, we) || !aligned(bias, we) || !aligned(mean, 4) ||
        !aligned(rstd, 4))
        return IM2WIN_EALIGN;
    if (rows == 0)
        return IM2WIN_OK;
    const Buf in[3] = {{x, ((rows - 1) * x_stride + C) * e}, {weight, C * we}, {bias, C * we}};
    const Buf out[3] = {{y, rows * C * e}, {mean, rows * 4}, {rstd, rows * 4}};
    int rc;
    Extents ext;
    if ((rc = ext.check(in, 3)) || (rc = ext.check(out, 3)))
        return rc;
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i)
            if (meet(out[o], in[i]) && !(o == 0 && i == 0 && x == y && x_stride == C))
                return IM2WIN_EOVERLAP;
        for (int i = 0; i < o; ++i)
            if (meet(out[o], out[i]))
                return IM2WIN_EOVERLAP;
    }
    if ((rc = check_device()))
        return rc;
    return launch_status(
        launch_norm_forward(x, weight, bias, y, mean, rstd, rows, C, x_stride, eps, dt, wdt, (hipStream_t)hip_stream));
}

int64_t seq_layer_norm_workspace_bytes(int64_t rows, int64_t C)
{
    if (rows < 0 || C <= 0)
        return IM2WIN_EINVAL;
    if (rows > INT32_MAX || C >= (int64_t)1 << 24)
        return IM2WIN_ERANGE;
    return pad256(norm_partial_rows(rows, C) * 2 * C * 4);
}

int seq_layer_norm_backward(const void *dy, const void *x, const void *weight, const float *mean, const float *rstd,
                            void *dx, void *dweight, void *dbias, void *ws, int64_t ws_bytes, int64_t rows, int64_t C,
                            int64_t dy_stride, int64_t x_stride, im2win_dtype_t dt, im2win_dtype_t wdt,
                            void *hip_stream)
{
    if (!known(dt) || (wdt != dt && wdt != IM2WIN_F32) || rows < 0 || C <= 0 || x_stride < C || dy_stride < C)
        return IM2WIN_EINVAL;
    if (!weight || !dweight || !dbias || !ws || (rows > 0 && (!dy || !x || !mean || !rstd || !dx)))
        return IM2WIN_EINVAL;
    if (rows > INT32_MAX || C >= (int64_t)1 << 24 || too_far(rows, x_stride) || too_far(rows, dy_stride))
        return IM2WIN_ERANGE;
    const int64_t e = elt(dt), we = elt(wdt);
    if (!aligned(dy, e) || !aligned(x, e) || !aligned(dx, e) || !aligned(weight, we) || !aligned(dweight, we) ||
        !aligned(dbias, we) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(ws, 16))
        return IM2WIN_EALIGN;
    if (ws_bytes < 0)
        return IM2WIN_EWORKSPACE;
    const int64_t reach = rows > 0 ? rows - 1 : 0, any = rows > 0;
    const Buf in[5] = {{dy, any * (reach * dy_stride + C) * e},
                       {x, any * (reach * x_stride + C) * e},
                       {weight, C * we},
                       {mean, rows * 4},
                       {rstd, rows * 4}};
    const Buf out[4] = {{dx, rows * C * e}, {dweight, C * we}, {dbias, C * we}, {ws, ws_bytes}};
    int rc;
    Extents ext;
    if ((rc = ext.check(in, 5)) || (rc = ext.check(out, 4)))
        return rc;
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 5; ++i)
            if (meet(out[o], in[i]))
                return IM2WIN_EOVERLAP;
        for (int i = 0; i < o; ++i)
            if (meet(out[o], out[i]))
                return IM2WIN_EOVERLAP;
    }
    if (ws_bytes < seq_layer_norm_workspace_bytes(rows, C))
        return IM2WIN_EWORKSPACE;
    if ((rc = check_device()))
        return rc;
    return launch_status(launch_norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, (float *)ws, rows, C,
                                              dy_stride, x_stride, dt, wdt, (hipStream_t)hip_stream));
}

static int check_bias(int64_t H, int64_t buckets, int64_t R, int two_sided)
{
    if (H <= 0 || buckets <= 0 || R <= 0 || (two_sided && buckets % 2))
        return IM2WIN_EINVAL;
    const int64_t m = two_sided ? buckets / 2 : buckets;
    if (m < 2 || R <= m / 2)
        return IM2WIN_EINVAL;
    if (m > kMaxBuckets || R > SEQ_BIAS_RANGE || H >= 1 << 16)
        return IM2WIN_ERANGE;
    return IM2WIN_OK;
}

int64_t seq_rel_bias_bucket(int64_t d, int64_t buckets, int64_t R, int two_sided)
{
    if (const int rc = check_bias(1, buckets, R, two_sided))
        return rc;
    const Buckets bk = make_buckets(buckets, R, two_sided);
    d = d < -R ? -R : d > R ? R : d;
    const int64_t n = d < 0 ? -d : two_sided ? d : 0;
    int64_t b = n;
    if (n >= bk.e)
        for (b = bk.e; bk.from[b - bk.e + 1] <= n;)
            ++b;
    return two_sided && d > 0 ? b + bk.m : b;
}

int seq_rel_bias_forward(const void *table, float *strip, int64_t H, int64_t buckets, int64_t R, int two_sided,
                         im2win_dtype_t dt, void *hip_stream)
{
    if (!table || !strip || !known(dt))
        return IM2WIN_EINVAL;
    int rc;
    if ((rc = check_bias(H, buckets, R, two_sided)))
        return rc;
    if (!aligned(table, elt(dt)) || !aligned(strip, 4))
        return IM2WIN_EALIGN;
    const Buf b[2] = {{table, buckets * H * elt(dt)}, {strip, H * (2 * R + 1) * 4}};
    if ((rc = Extents().check(b, 2)))
        return rc;
    if (meet(b[0], b[1]))
        return IM2WIN_EOVERLAP;
    if ((rc = check_device()))
        return rc;
    return launch_status(
        launch_bias_forward(make_buckets(buckets, R, two_sided), table, strip, H, dt, (hipStream_t)hip_stream));
}

int seq_rel_bias_backward(const float *dstrip, void *dtable, int64_t n, int64_t H, int64_t buckets, int64_t R,
                          int two_sided, im2win_dtype_t dt, void *hip_stream)
{
    if ((!dstrip && n > 0) || !dtable || !known(dt) || n < 0)
        return IM2WIN_EINVAL;
    int rc;
    if ((rc = check_bias(H, buckets, R, two_sided)))
        return rc;
    if (n >= 1 << 16)
        return IM2WIN_ERANGE;
    if (!aligned(dstrip, 4) || !aligned(dtable, elt(dt)))
        return IM2WIN_EALIGN;
    const Buf b[2] = {{dstrip, n * H * (2 * R + 1) * 4}, {dtable, buckets * H * elt(dt)}};
    if ((rc = Extents().check(b, 2)))
        return rc;
    if (meet(b[0], b[1]))
        return IM2WIN_EOVERLAP;
    if ((rc = check_device()))
        return rc;
    return launch_status(
        launch_bias_backward(make_buckets(buckets, R, two_sided), dstrip, dtable, n, H, dt, (hipStream_t)hip_stream));
}

int64_t seq_attention_workspace_bytes(const seq_attention_t *a, int backward)
{
    if (const int rc = check_dims(a, backward != 0))
        return rc;
    return sizes_of(a, backward != 0).total;
}

static int attention(const seq_attention_t *a, const void *dout, const void *q, const void *k, const void *v,
                     const void *out, const float *lse, void *dq, void *dk, void *dv, float *dstrip, void *ws,
                     int64_t ws_bytes, void *hip_stream, bool backward)
{
    int rc;
    if ((rc = check_dims(a, backward)) && rc != IM2WIN_EOVERLAP)
        return rc;
    const int late = rc;
    const bool nq = a->B > 0 && a->Lq > 0, nk = a->B > 0 && a->Lk > 0;
    if ((nq && (!q || !out || !lse)) || (nk && (!k || !v)) || (a->R && !a->strip) ||
        (backward && ((nq && (!dout || !dq)) || (nk && (!dk || !dv)))))
        return IM2WIN_EINVAL;
    if (!a->q_doc != !a->k_doc && nq && nk)
        return IM2WIN_EINVAL;
    const int64_t e = elt(a->dt);
    const bool al = aligned(q, 16) && aligned(k, 16) && aligned(v, 16) && aligned(out, 16) && aligned(lse, 4) &&
                    aligned(dout, 16) && aligned(dq, 16) && aligned(dk, 16) && aligned(dv, 16) && aligned(dstrip, 4) &&
                    aligned(ws, 16) && aligned(a->strip, 4) && aligned(a->kv_len, 4) && aligned(a->prefix, 4) &&
                    aligned(a->q_doc, 4) && aligned(a->k_doc, 4) &&
                    strides_aligned(a->q_stride, a->B, a->Lq, a->H, e) &&
                    strides_aligned(a->k_stride, a->B, a->Lk, a->Hkv, e) &&
                    strides_aligned(a->v_stride, a->B, a->Lk, a->Hkv, e) &&
                    strides_aligned(a->out_stride, a->B, a->Lq, a->H, e) &&
                    (!backward || (strides_aligned(a->dout_stride, a->B, a->Lq, a->H, e) &&
                                   strides_aligned(a->dq_stride, a->B, a->Lq, a->H, e) &&
                                   strides_aligned(a->dk_stride, a->B, a->Lk, a->Hkv, e) &&
                                   strides_aligned(a->dv_stride, a->B, a->Lk, a->Hkv, e)));
    if (!al)
        return IM2WIN_EALIGN;
    const Sizes s = sizes_of(a, backward);
    if (ws_bytes < 0 || (!ws && s.total > 0))
        return IM2WIN_EWORKSPACE;
    const Operand oq{q, a->B, a->Lq, a->H, a->D, e, a->q_stride}, ok{k, a->B, a->Lk, a->Hkv, a->D, e, a->k_stride},
        ov{v, a->B, a->Lk, a->Hkv, a->D, e, a->v_stride}, oo{out, a->B, a->Lq, a->H, a->D, e, a->out_stride},
        odo{dout, a->B, a->Lq, a->H, a->D, e, a->dout_stride}, odq{dq, a->B, a->Lq, a->H, a->D, e, a->dq_stride},
        odk{dk, a->B, a->Lk, a->Hkv, a->D, e, a->dk_stride}, odv{dv, a->B, a->Lk, a->Hkv, a->D, e, a->dv_stride};
    const int64_t strip_bytes = a->R ? a->H * (2 * a->R + 1) * 4 : 0, lse_bytes = a->B * a->H * a->Lq * 4;
    const Operand *ins[6] = {&oq, &ok, &ov, &oo, &odo, nullptr}, *outs[3] = {&oo, nullptr, nullptr};
    int n_in = 3, n_out = 1;
    if (backward) {
        n_in = 5, n_out = 3;
        outs[0] = &odq, outs[1] = &odk, outs[2] = &odv;
    }
    const Buf small[5] = {{a->strip, strip_bytes},
                          {a->kv_len, a->kv_len ? a->B * 4 : 0},
                          {a->prefix, a->causal && a->prefix ? a->B * 4 : 0},
                          {a->q_doc, a->q_doc ? a->B * a->Lq * 4 : 0},
                          {a->k_doc, a->k_doc ? a->B * a->Lk * 4 : 0}};
    const Buf flat[3] = {{lse, lse_bytes}, {dstrip, backward && dstrip ? strip_bytes : 0}, {ws, ws_bytes}};
    Extents ext;
    for (int i = 0; i < n_in; ++i) {
        const Buf b{ins[i]->p, ins[i]->bytes()};
        if ((rc = ext.check(&b, 1)))
            return rc;
    }
    for (int i = 0; i < n_out; ++i) {
        const Buf b{outs[i]->p, outs[i]->bytes()};
        if ((rc = ext.check(&b, 1)))
            return rc;
    }
    if ((rc = ext.check(small, 5)) || (rc = ext.check(flat, 3)))
        return rc;
    if (late)
        return late;
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (clash(*outs[i], *ins[j]))
                return IM2WIN_EOVERLAP;
        for (int j = 0; j < i; ++j)
            if (clash(*outs[i], *outs[j]))
                return IM2WIN_EOVERLAP;
        const Buf b{outs[i]->p, outs[i]->bytes()};
        for (const Buf &m : small)
            if (meet(b, m))
                return IM2WIN_EOVERLAP;
        for (const Buf &m : flat)
            if (meet(b, m))
                return IM2WIN_EOVERLAP;
    }
    for (int i = 0; i < 3; ++i) {
        if (i == 0 && backward)  // lse is read there
            continue;
        for (int j = 0; j < n_in; ++j)
            if (meet(flat[i], Buf{ins[j]->p, ins[j]->bytes()}))
                return IM2WIN_EOVERLAP;
        for (const Buf &m : small)
            if (meet(flat[i], m))
                return IM2WIN_EOVERLAP;
        for (int j = 0; j < i; ++j)
            if (meet(flat[i], flat[j]))
                return IM2WIN_EOVERLAP;
    }
    if (ws_bytes < s.total)
        return IM2WIN_EWORKSPACE;
    if ((rc = check_device()))
        return rc;
    const hipStream_t st = (hipStream_t)hip_stream;
    AttnArgs r = make_args(a);
    r.q = (const char *)q, r.k = (const char *)k, r.v = (const char *)v;
    if (!backward && !nq)
        return IM2WIN_OK;
    if (!nk)  // no key: the documents' ids are not read either
        r.q_doc = r.k_doc = nullptr;
    if (r.q_doc || ws) {
        seq_attention_t d = *a;
        d.q_doc = r.q_doc;
        if ((rc = place(&r, &d, s, ws, st)))
            return rc;
    }
    if (!backward) {
        r.out = (char *)out, r.lse = const_cast<float *>(lse);
        return launch_status(launch_attn_forward(r, a->dt, st));
    }
    r.o = (const char *)out, r.dout = (const char *)dout, r.lse = const_cast<float *>(lse);
    r.dq = (char *)dq, r.dk = (char *)dk, r.dv = (char *)dv;
    set_strides(odo, r.do_sb, r.do_st, r.do_sh);
    set_strides(odq, r.dq_sb, r.dq_st, r.dq_sh);
    set_strides(odk, r.dk_sb, r.dk_st, r.dk_sh);
    set_strides(odv, r.dv_sb, r.dv_st, r.dv_sh);
    return launch_status(launch_attn_backward(r, a->dt, a->R ? dstrip : nullptr, st));
}

int seq_attention_forward(const seq_attention_t *a, const void *q, const void *k, const void *v, void *out, float *lse,
                          void *ws, int64_t ws_bytes, void *hip_stream)
{
    return attention(a, nullptr, q, k, v, out, lse, nullptr, nullptr, nullptr, nullptr, ws, ws_bytes, hip_stream, false);
}

int seq_attention_backward(const seq_attention_t *a, const void *dout, const void *q, const void *k, const void *v,
                           const void *out, const float *lse, void *dq, void *dk, void *dv, float *dstrip, void *ws,
                           int64_t ws_bytes, void *hip_stream)
{
    return attention(a, dout, q, k, v, out, lse, dq, dk, dv, dstrip, ws, ws_bytes, hip_stream, true);
}

}  // extern "C"
