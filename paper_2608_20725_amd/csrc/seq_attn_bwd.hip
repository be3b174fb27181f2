// Attention backward.  The scores are computed again from q and k, the
// probabilities from the forward pass's row statistics:
//   P = exp(s - lse),  dP = dout v^T,  dS = P (dP - delta),  delta = dout.out
//   dv = P^T dout,  dk = scale dX^T q,  dq = scale dX k,  dX = dS (1 - tanh^2).
// Two kernels, each with its own held side, so that every gradient has one
// owner and no atomics: attn_dkdv holds 128 keys and streams the queries of
// all heads that share them (4 products a pair), attn_dq holds 128 queries
// and streams keys (3 products, two of them the same as there).  The strip's
// gradient is summed along the diagonals in attn_dq.
//
// fp16 keeps 5 exponent bits: P is multiplied by 2^14 and dS by a power of
// two that brings its bound 2 max|dout_i| max|v_j| to at most 2^15, so that
// the small probabilities of long rows and the gradients of a scaled loss
// both stay normal numbers; the fp32 sums are divided again.
#include "seq_attn.hpp"

namespace im2win {
namespace {

constexpr int kThreads = 64 * kWaves;

template <class Op>
constexpr float p_shift() { return 0.0f; }
template <>
constexpr float p_shift<F16Op>() { return 14.0f; }

// The power of two that dS of a head group is multiplied by.
template <class Op>
__device__ inline float ds_scale(const AttnArgs &a, int b, int hk)
{
    if constexpr (sizeof(typename Op::elem) == 2 && p_shift<Op>() > 0) {
        const uint32_t *n = a.norms + ((int64_t)b * a.Hkv + hk) * 2;
        const float bound = 2.0f * __uint_as_float(n[0]) * __uint_as_float(n[1]);
        const float e = bound > 0 ? floorf(15.0f - __log2f(bound) - 0.01f) : 0.0f;
        return exp2f(fminf(fmaxf(e, -40.0f), 40.0f));
    }
    return 1.0f;
}

// ---- row statistics ----

__global__ __launch_bounds__(kThreads) void clear_words(uint32_t *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
        p[i] = 0;
}

template <class Op>
__device__ inline void load8(const char *p, float *f)
{
    const typename Op::v8 v = *(const typename Op::v8 *)p;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] = (float)v[e];
}

__device__ inline float sum16(float v)
{
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1)
        v += __shfl_xor(v, m);
    return v;
}

// Raises *to to the largest finite value of v over the workgroup.
__device__ inline void raise(uint32_t *to, float v)
{
    v = v < INFINITY ? v : 0.0f;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        v = fmaxf(v, __shfl_xor(v, m));
    if ((threadIdx.x & 63) == 0)
        atomicMax(to, __float_as_uint(v));  // a maximum: the same in any order
}

// 16 lanes a row: {lse*log2(e), dout.out} and, fp16, the largest |dout|.
template <class Op>
__global__ __launch_bounds__(kThreads) void row_stats(AttnArgs a)
{
    const uint32_t bh = blockIdx.x / a.tiles, t = blockIdx.x - bh * a.tiles;
    const int b = bh / a.H, hq = bh - b * a.H;
    const int i = t * (kThreads / 16) + (threadIdx.x >> 4), d = (threadIdx.x & 15) * 8;
    float f[8], g[8], dot = 0, sq = 0;
    if (i < a.Lq && d < a.D) {
        load8<Op>(a.dout + b * a.do_sb + hq * a.do_sh + (int64_t)i * a.do_st + d * sizeof(typename Op::elem), f);
        load8<Op>(a.o + b * a.o_sb + hq * a.o_sh + (int64_t)i * a.o_st + d * sizeof(typename Op::elem), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            dot += f[e] * g[e];
            sq += f[e] * f[e];
        }
    }
    dot = sum16(dot);
    sq = sum16(sq);
    bool some = false;
    if (i < a.Lq) {
        const int64_t at = (int64_t)bh * a.Lq + i;
        const float l = a.lse[at];
        some = l != -INFINITY;
        if (d == 0)
            a.stat[at] = make_float2(some ? l * kLog2e : INFINITY, dot);
    }
    if constexpr (p_shift<Op>() > 0)
        raise(a.norms + ((int64_t)b * a.Hkv + hq / a.G) * 2, some ? sqrtf(sq) : 0.0f);
}

// fp16: the largest |v_j| of each key/value head.
template <class Op>
__global__ __launch_bounds__(kThreads) void value_norms(AttnArgs a)
{
    const uint32_t bh = blockIdx.x / a.tiles, t = blockIdx.x - bh * a.tiles;
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int j = t * (kThreads / 16) + (threadIdx.x >> 4), d = (threadIdx.x & 15) * 8;
    float f[8], sq = 0;
    const bool in = j < keys_of(a, b) && (!a.k_doc || a.k_doc[(int64_t)b * a.Lk + j] >= 0);
    if (in && d < a.D) {
        load8<Op>(a.v + b * a.v_sb + hk * a.v_sh + (int64_t)j * a.v_st + d * sizeof(typename Op::elem), f);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sq += f[e] * f[e];
    }
    raise(a.norms + ((int64_t)b * a.Hkv + hk) * 2 + 1, sqrtf(sum16(sq)));
}

// ---- what both kernels do with a 32 x 32 tile of scores ----

// Scores (times log2 e) of products q.k, without the bias; slope: 1 - tanh^2
// where they are capped.
__device__ inline void to_scores(f32x16_acc &s, f32x16_acc &slope, const ScoreArgs &c)
{
    if (c.cap) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float t = fast_tanh(s[r] * c.c1);
            slope[r] = 1.0f - t * t;
            s[r] = c.c2 * t;
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] *= c.c1;
    }
}

template <class Op, int DP>
struct Bwd {
    typedef Tile<Op, DP> T;
    static constexpr int kRows = OpInfo<Op>::kIs32 ? 32 : 64;  // streamed tokens a tile
    static constexpr int kSub = kRows / 32;
    static constexpr int kTileBytes = kRows * T::kRowBytes;
};

// ---- dk, dv: a key per lane ----
template <class Op, int DP>
__global__ __launch_bounds__(kThreads) void attn_dkdv(AttnArgs a)
{
    typedef Bwd<Op, DP> W;
    typedef Tile<Op, DP> T;
    extern __shared__ __align__(16) char lds[];
    char *const tq = lds, *const tdo = lds + W::kTileBytes;
    float *const strip = (float *)(lds + 2 * W::kTileBytes);
    __shared__ float s_lse[W::kRows], s_delta[W::kRows];
    __shared__ int s_doc[W::kRows];
    __shared__ int shared_first[kWaves], shared_lo[kWaves], shared_hi[kWaves];

    uint32_t kt;
    const uint32_t bh = work_item((uint32_t)(a.B * a.Hkv) * a.tiles, a.tiles, &kt);
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = threadIdx.x >> 6;
    const int j = kt * kHeld + wave * 32 + (lane & 31);  // this lane's key
    const bool in = j < a.Lk;
    const int n = keys_of(a, b), off = first_pos(a, n);

    // queries from `first` on see this key (with documents: of the same one)
    int first = 0, doc = 0;
    if (a.causal && !(a.prefix && j < a.prefix[b]))
        first = max(j - off, 0);
    if (j >= n)
        first = INT32_MAX;
    if (a.k_doc) {
        doc = in ? a.k_doc[(int64_t)b * a.Lk + j] : -1;
        if (doc < 0)
            first = INT32_MAX;
    }
    const bool live = first < a.Lq;
    const int least = wave_min(first), most = wave_max(first);
    const int jlo = kt * kHeld + wave * 32, jhi = jlo + 31;
    const int dlo = wave_min(live ? doc : INT32_MAX), dhi = wave_max(live ? doc : -1);
    if (lane == 0) {
        shared_first[wave] = least;
        shared_lo[wave] = dlo;
        shared_hi[wave] = dhi;
    }
    __syncthreads();
    int wg_first = INT32_MAX, wg_lo = INT32_MAX, wg_hi = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        wg_first = min(wg_first, shared_first[w]);
        wg_lo = min(wg_lo, shared_lo[w]);
        wg_hi = max(wg_hi, shared_hi[w]);
    }

    const bool held = in && j < n;
    typename Op::v8 kf[DP / 16], vf[DP / 16];
    T::held(kf, a.k + b * a.k_sb + hk * a.k_sh + (int64_t)j * a.k_st, held, h, a.D);
    T::held(vf, a.v + b * a.v_sb + hk * a.v_sh + (int64_t)j * a.v_st, held, h, a.D);
    f32x16_acc dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            dk[t][r] = dv[t][r] = 0;

    const ScoreArgs sc = score_args(a);
    const float dss = ds_scale<Op>(a, b, hk);
    const float f = dss * exp2f(-p_shift<Op>());  // dS*dss = P' * (f*dP - f*delta)

    for (int g = 0; g < a.G; ++g) {
        const int hq = hk * a.G + g;
        if (a.R) {
            __syncthreads();
            for (int t = threadIdx.x; t < 2 * a.R + 1; t += kThreads)
                strip[t] = a.strip[(int64_t)hq * (2 * a.R + 1) + t] * kLog2e;
        }
        const char *qp = a.q + b * a.q_sb + hq * a.q_sh, *dop = a.dout + b * a.do_sb + hq * a.do_sh;
        const float2 *stat = a.stat + ((int64_t)b * a.H + hq) * a.Lq;
        for (int q0 = wg_first / W::kRows * W::kRows; q0 < a.Lq; q0 += W::kRows) {
            DocRange dr = {0, 0, 0, 0};
            if (a.k_doc) {
                dr = a.q_range[(int64_t)b * ((a.Lq + kDocTile - 1) / kDocTile) + q0 / kDocTile];
                if (!(dr.lo <= wg_hi && dr.hi >= wg_lo))
                    continue;
            }
            __syncthreads();
            T::template stage<W::kRows>(tq, qp + (int64_t)q0 * a.q_st, a.q_st, a.Lq - q0, a.D);
            T::template stage<W::kRows>(tdo, dop + (int64_t)q0 * a.do_st, a.do_st, a.Lq - q0, a.D);
            if (threadIdx.x < W::kRows) {
                const int i = q0 + threadIdx.x;
                float2 v = make_float2(INFINITY, 0);
                if (i < a.Lq)
                    v = stat[i];
                s_lse[threadIdx.x] = v.x - p_shift<Op>();
                s_delta[threadIdx.x] = v.y * f;
                if (a.k_doc)
                    s_doc[threadIdx.x] = i < a.Lq ? a.q_doc[(int64_t)b * a.Lq + i] : -1;
            }
            __syncthreads();
            if (q0 + W::kRows <= least || (a.k_doc && !(dr.lo <= dhi && dr.hi >= dlo)))
                continue;
            const bool docs_differ = a.k_doc && (dr.mixed || dlo != dhi || dr.lo != dlo);
            const bool partial = q0 < most || docs_differ;
#pragma unroll
            for (int t = 0; t < W::kSub; ++t) {
                f32x16_acc s, dp, slope;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = dp[r] = 0;
#pragma unroll
                for (int st = 0; st < DP / 16; ++st) {
                    s = Op::mfma(T::row_frag(tq, 32 * t + (lane & 31), st, h), kf[st], s);
                    dp = Op::mfma(T::row_frag(tdo, 32 * t + (lane & 31), st, h), vf[st], dp);
                }
                to_scores(s, slope, sc);
                const int i0 = q0 + 32 * t;
                if (a.R) {
                    const int dmin = jlo - (i0 + 31 + off), dmax = jhi - (i0 + off);
                    if (dmax <= -a.R || dmin >= a.R) {
                        const float far = strip[dmin >= a.R ? 2 * a.R : 0];
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            s[r] += far;
                    } else {
                        const int d0 = j - (i0 + 4 * h + off);
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            s[r] += strip[min(max(d0 - reg_row(r), -a.R), a.R) + a.R];
                    }
                }
                bool out[16];
                const int lim = first == INT32_MAX ? INT32_MAX : first - i0 - 4 * h;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    out[r] = partial && (reg_row(r) < lim || (docs_differ && s_doc[32 * t + reg_row(r) + 4 * h] != doc));
                    const float delta = s_delta[32 * t + reg_row(r) + 4 * h];
                    float p = __builtin_amdgcn_exp2f(s[r] - s_lse[32 * t + reg_row(r) + 4 * h]);
                    float ds = p * (dp[r] * f - delta);
                    if (sc.cap)
                        ds *= slope[r];
                    if (partial) {
                        p += 0.0f * delta;  // a dout that is not finite reaches dv through p
                        p = out[r] ? 0.0f : p;
                        ds = out[r] ? 0.0f : ds;
                    }
                    s[r] = p;
                    dp[r] = ds;
                }
                uint32_t bad = 0;
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    const typename Op::v8 p = pack8<Op>(s, 8 * ks), ds = pack8<Op>(dp, 8 * ks);
#pragma unroll
                    for (int dt = 0; dt < DP / 32; ++dt) {
                        typename Op::v8 x = T::col_frag(tdo, 32 * t + 16 * ks, dt, lane);
                        typename Op::v8 y = T::col_frag(tq, 32 * t + 16 * ks, dt, lane);
                        if (partial) {  // a left-out pair's zero times infinity or NaN must stay zero
                            x = finite<Op>(x, bad);
                            y = finite<Op>(y, bad);
                        }
                        dv[dt] = Op::mfma(x, p, dv[dt]);
                        dk[dt] = Op::mfma(y, ds, dk[dt]);
                    }
                }
            }
        }
    }
    if (!in)
        return;
    store_row<Op, DP>(a.dk + b * a.dk_sb + hk * a.dk_sh + (int64_t)j * a.dk_st, dk, a.scale / dss, h, a.D);
    store_row<Op, DP>(a.dv + b * a.dv_sb + hk * a.dv_sh + (int64_t)j * a.dv_st, dv, exp2f(-p_shift<Op>()), h, a.D);
}

// ---- dq (and the strip's gradient): a query per lane ----
template <class Op, int DP>
__global__ __launch_bounds__(kThreads) void attn_dq(AttnArgs a, int want_strip)
{
    typedef Bwd<Op, DP> W;
    typedef Tile<Op, DP> T;
    extern __shared__ __align__(16) char lds[];
    char *const tk = lds, *const tv = lds + W::kTileBytes;
    float *const strip = (float *)(lds + 2 * W::kTileBytes);
    const int width = 2 * a.R + 1;
    __shared__ int kdoc[W::kRows];
    __shared__ int shared_most[kWaves], shared_lo[kWaves], shared_hi[kWaves];

    uint32_t qt;
    const uint32_t bh = work_item((uint32_t)(a.B * a.H) * a.tiles, a.tiles, &qt);
    qt = a.tiles - 1 - qt;
    const int b = bh / a.H, hq = bh - b * a.H, hk = hq / a.G;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = threadIdx.x >> 6;
    const int i = qt * kHeld + wave * 32 + (lane & 31);
    const bool live = i < a.Lq;
    const int n = keys_of(a, b);
    const int pos = i + first_pos(a, n);
    int lim = n, doc = 0;
    if (a.causal)
        lim = min(n, max(pos + 1, a.prefix ? a.prefix[b] : 0));
    if (a.q_doc) {
        doc = live ? a.q_doc[(int64_t)b * a.Lq + i] : -1;
        if (doc < 0)
            lim = 0;
    }
    if (!live || lim < 0)
        lim = 0;
    const int most = wave_max(lim), least = wave_min(lim);
    const int plo = wave_min(pos), phi = wave_max(pos);
    const int dlo = wave_min(lim > 0 ? doc : INT32_MAX), dhi = wave_max(lim > 0 ? doc : -1);
    // each half wave has a strip of gradients of its own: the 32 lanes that
    // add in one instruction hold 32 different distances, so nothing is
    // summed in an order that could change
    float *const grad = strip + width * (1 + 2 * wave + h);
    float far_lo = 0, far_hi = 0;
    if (a.R)
        for (int t = threadIdx.x; t < width; t += kThreads) {
            strip[t] = a.strip[(int64_t)hq * width + t] * kLog2e;
            if (want_strip)
#pragma unroll
                for (int w = 1; w <= 2 * kWaves; ++w)
                    strip[w * width + t] = 0;
        }
    if (lane == 0) {
        shared_most[wave] = most;
        shared_lo[wave] = dlo;
        shared_hi[wave] = dhi;
    }
    __syncthreads();
    int wg_most = 0, wg_lo = INT32_MAX, wg_hi = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        wg_most = max(wg_most, shared_most[w]);
        wg_lo = min(wg_lo, shared_lo[w]);
        wg_hi = max(wg_hi, shared_hi[w]);
    }

    typename Op::v8 qf[DP / 16], dof[DP / 16];
    T::held(qf, a.q + b * a.q_sb + hq * a.q_sh + (int64_t)i * a.q_st, live, h, a.D);
    T::held(dof, a.dout + b * a.do_sb + hq * a.do_sh + (int64_t)i * a.do_st, live, h, a.D);
    float2 st = make_float2(INFINITY, 0);
    if (live)
        st = a.stat[((int64_t)b * a.H + hq) * a.Lq + i];
    const float dss = ds_scale<Op>(a, b, hk);
    const float lse = st.x - p_shift<Op>(), delta = st.y * dss * exp2f(-p_shift<Op>());
    // The matrix cores' 16-bit products come out low by 1 % of an ulp in the
    // mean (measured: -9e-9 at |dP| of 8), which sums over the thousands of
    // pairs of a bucket.  Every second query holds -dout, so that what the
    // queries add to a distance is off in both directions.
    const float f = dss * exp2f(-p_shift<Op>()) * (lane & 1 ? -1.0f : 1.0f);
    if (lane & 1)
#pragma unroll
        for (int x = 0; x < DP / 16; ++x)
            dof[x] = -dof[x];
    f32x16_acc dq[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            dq[t][r] = 0;
    const char *kp = a.k + b * a.k_sb + hk * a.k_sh, *vp = a.v + b * a.v_sb + hk * a.v_sh;
    const ScoreArgs sc = score_args(a);

    for (int k0 = 0; k0 < wg_most; k0 += W::kRows) {
        DocRange dr = {0, 0, 0, 0};
        if (a.q_doc) {
            dr = a.k_range[(int64_t)b * ((a.Lk + kDocTile - 1) / kDocTile) + k0 / kDocTile];
            if (!(dr.lo <= wg_hi && dr.hi >= wg_lo))
                continue;
        }
        __syncthreads();
        T::template stage<W::kRows>(tk, kp + (int64_t)k0 * a.k_st, a.k_st, n - k0, a.D);
        T::template stage<W::kRows>(tv, vp + (int64_t)k0 * a.v_st, a.v_st, n - k0, a.D);
        if (a.q_doc && threadIdx.x < W::kRows)
            kdoc[threadIdx.x] = k0 + (int)threadIdx.x < n ? a.k_doc[(int64_t)b * a.Lk + k0 + threadIdx.x] : -1;
        __syncthreads();
        if (k0 >= most || (a.q_doc && !(dr.lo <= dhi && dr.hi >= dlo)))
            continue;
        const bool docs_differ = a.q_doc && (dr.mixed || dlo != dhi || dr.lo != dlo);
        const bool partial = k0 + W::kRows > least || docs_differ;
#pragma unroll
        for (int t = 0; t < W::kSub; ++t) {
            f32x16_acc s, dp, slope;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[r] = dp[r] = 0;
#pragma unroll
            for (int x = 0; x < DP / 16; ++x) {
                s = Op::mfma(T::row_frag(tk, 32 * t + (lane & 31), x, h), qf[x], s);
                dp = Op::mfma(T::row_frag(tv, 32 * t + (lane & 31), x, h), dof[x], dp);
            }
            to_scores(s, slope, sc);
            const int j0 = k0 + 32 * t, d0 = j0 + 4 * h - pos;
            const bool far = a.R && (j0 + 31 - plo <= -a.R || j0 - phi >= a.R);
            if (a.R) {
                if (far) {
                    const float v = strip[j0 - phi >= a.R ? 2 * a.R : 0];
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] += v;
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] += strip[min(max(d0 + reg_row(r), -a.R), a.R) + a.R];
                }
            }
            const int last = lim - j0 - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(s[r] - lse);
                float ds = p * (dp[r] * f - delta);
                if (partial)
                    ds = reg_row(r) >= last || (docs_differ && kdoc[32 * t + reg_row(r) + 4 * h] != doc) ? 0.0f : ds;
                dp[r] = ds;
            }
            if (want_strip) {
                if (far) {
                    float v = 0;
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        v += dp[r];
                    if (j0 - phi >= a.R)
                        far_hi += v;
                    else
                        far_lo += v;
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int d = d0 + reg_row(r);
                        far_lo += d <= -a.R ? dp[r] : 0.0f;
                        far_hi += d >= a.R ? dp[r] : 0.0f;
                        if (d > -a.R && d < a.R)
                            __hip_atomic_fetch_add(grad + d + a.R, dp[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
                    }
                }
            }
            if (sc.cap)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    dp[r] *= slope[r];
            uint32_t bad = 0;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const typename Op::v8 ds = pack8<Op>(dp, 8 * ks);
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt) {
                    typename Op::v8 x = T::col_frag(tk, 32 * t + 16 * ks, dt, lane);
                    if (partial)
                        x = finite<Op>(x, bad);
                    dq[dt] = Op::mfma(x, ds, dq[dt]);
                }
            }
        }
    }
    if (live)
        store_row<Op, DP>(a.dq + b * a.dq_sb + hq * a.dq_sh + (int64_t)i * a.dq_st, dq, a.scale / dss, h, a.D);
    if (!want_strip)
        return;
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        far_lo += __shfl_xor(far_lo, m);
        far_hi += __shfl_xor(far_hi, m);
    }
    __syncthreads();
    if (lane == 0) {  // the ends of the strip are only summed in registers
        strip[width * (1 + 2 * wave)] = far_lo;
        strip[width * (1 + 2 * wave) + 2 * a.R] = far_hi;
    }
    __syncthreads();
    float *out = a.part + (((int64_t)hq * a.B + b) * a.tiles + qt) * width;
    for (int t = threadIdx.x; t < width; t += kThreads) {
        float v = 0;
#pragma unroll
        for (int w = 1; w <= 2 * kWaves; ++w)
            v += strip[w * width + t];
        out[t] = v / dss;
    }
}

// dstrip[h][x]: the sum of `n` partial strips, 64 entries a workgroup, each
// by four lanes that take every fourth strip.
__global__ __launch_bounds__(kThreads) void strip_reduce(const float *__restrict__ part, float *__restrict__ dstrip,
                                                         int32_t n, int32_t width)
{
    __shared__ float s[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6, h = blockIdx.y;
    float v = 0;
    if (c < width)
        for (int r = k; r < n; r += 4)
            v += part[((int64_t)h * n + r) * width + c];
    s[k][threadIdx.x & 63] = v;
    __syncthreads();
    if (k == 0 && c < width)
        dstrip[(int64_t)h * width + c] =
            (s[0][threadIdx.x] + s[1][threadIdx.x]) + (s[2][threadIdx.x] + s[3][threadIdx.x]);
}

template <class Op, int DP>
hipError_t run(const AttnArgs &a, float *dstrip, hipStream_t st)
{
    typedef Bwd<Op, DP> W;
    const int width = 2 * a.R + 1;
    AttnArgs b = a;
    hipError_t e;
    if constexpr (p_shift<Op>() > 0) {
        const int64_t words = (int64_t)a.B * a.Hkv * 2;
        if (words)
            clear_words<<<(uint32_t)((words + kThreads - 1) / kThreads < 256 ? (words + kThreads - 1) / kThreads : 256),
                          kThreads, 0, st>>>(a.norms, words);
        b.tiles = (a.Lk + kThreads / 16 - 1) / (kThreads / 16);
        if (a.B * b.tiles)
            value_norms<Op><<<(uint32_t)(a.B * a.Hkv) * b.tiles, kThreads, 0, st>>>(b);
    }
    b.tiles = (a.Lq + kThreads / 16 - 1) / (kThreads / 16);
    if (a.B * b.tiles)
        row_stats<Op><<<(uint32_t)(a.B * a.H) * b.tiles, kThreads, 0, st>>>(b);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;

    constexpr size_t kMost = 2 * W::kTileBytes + (2 * SEQ_BIAS_RANGE + 1) * 4;
    if ((e = hipFuncSetAttribute((const void *)attn_dkdv<Op, DP>, hipFuncAttributeMaxDynamicSharedMemorySize, kMost)) !=
            hipSuccess ||
        (e = hipFuncSetAttribute((const void *)attn_dq<Op, DP>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                 kMost + 2 * kWaves * (2 * SEQ_BIAS_RANGE + 1) * 4)) != hipSuccess)
        return e;
    b.tiles = (a.Lk + kHeld - 1) / kHeld;
    if (a.B * b.tiles)
        attn_dkdv<Op, DP><<<(uint32_t)(a.B * a.Hkv) * b.tiles, kThreads, 2 * W::kTileBytes + (a.R ? width * 4 : 0), st>>>(
            b);
    b.tiles = (a.Lq + kHeld - 1) / kHeld;
    if (a.B * b.tiles)
        attn_dq<Op, DP><<<(uint32_t)(a.B * a.H) * b.tiles, kThreads,
                          2 * W::kTileBytes + (a.R ? width * 4 * (dstrip ? 1 + 2 * kWaves : 1) : 0), st>>>(
            b, dstrip != nullptr);
    if (dstrip)
        strip_reduce<<<dim3((uint32_t)((width + 63) / 64), (uint32_t)a.H), kThreads, 0, st>>>(a.part, dstrip,
                                                                                           a.B * b.tiles, width);
    return hipGetLastError();
}

template <class Op>
hipError_t run_dim(const AttnArgs &a, float *dstrip, hipStream_t st)
{
    return a.D <= 32 ? run<Op, 32>(a, dstrip, st)
         : a.D <= 64 ? run<Op, 64>(a, dstrip, st)
         : a.D <= 96 ? run<Op, 96>(a, dstrip, st)
                     : run<Op, 128>(a, dstrip, st);
}

}  // namespace

int64_t attn_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D, int64_t R,
                        bool backward)
{
    if (!backward)
        return attn_few_rows(B, Lq, Lk, H, Hkv) ? attn_decode_part_bytes(dt, B, Lq, Lk, H, Hkv, D) : 0;
    if (R == 0)
        return 0;
    return B * H * ((Lq + kHeld - 1) / kHeld) * (2 * R + 1) * 4;
}

hipError_t launch_attn_backward(const AttnArgs &a, int dt, float *dstrip, hipStream_t st)
{
    return dt == IM2WIN_F32   ? run_dim<F32Op>(a, dstrip, st)
           : dt == IM2WIN_F16 ? run_dim<F16Op>(a, dstrip, st)
                              : run_dim<BF16Op>(a, dstrip, st);
}

}  // namespace im2win
