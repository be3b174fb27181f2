// Attention backward.  The scores are computed again from q and k, the
// probabilities from the forward pass's row statistics:
//   P = exp(s - lse),  dP = dout v^T,  dS = P (dP - delta),  delta = dout.out
//   dv = P^T dout,  dk = scale dX^T q,  dq = scale dX k,  dX = dS (1 - tanh^2).
// Two kernels, each with its own held side, so that every gradient has one
// owner: attn_dkdv holds 128 keys and streams the queries of
// all heads that share them (4 products a pair), attn_dq holds 128 queries
// and streams keys (3 products, two of them the same as there).  The strip's
// gradient is summed along the diagonals in attn_dq.  Bound by the matrix
// cores and, with a cap or a bias, by the vector operations of both kernels'
// scores, in attn_dq one score's after the other's (its mask is a branch for
// each): 2x4096 causal tokens, 32 query heads of 128 over 8, cap 30, bf16:
// 1280 us, of which attn_dkdv 803, attn_dq 505 and row_stats 27 when profiled.
//
// fp16 keeps 5 exponent bits: P is multiplied by 2^14 and dS by a power of
// two that brings its bound 2 max|dout_i| max|v_j| to at most 2^15, so that
// the small probabilities of long rows and the gradients of a scaled loss
// both stay normal numbers; the fp32 sums are divided again.
#include "seq_attn.hpp"

namespace im2win {
namespace {

constexpr int kThreads = 64 * kWaves;

// Rows of statistics a head has: whole tiles.
__host__ __device__ inline int stat_rows(int Lq) { return (Lq + 63) / 64 * 64; }

// Workgroups that share the keys of one query tile in attn_dq, as in the
// forward pass; a key costs more here, so shorter rows are worth it.  Measured,
// whole backward calls, one workgroup against split: bf16, 8 heads of 128, 1024
// tokens 81 -> 61 us; 16 heads of 64, 2048 tokens 112 -> 102 (causal 107 ->
// 92); fp32, 4 heads of 64, 256 tokens 79 -> 67.  Not split, 256 tiles of 1024
// keys in 16 bits: 73.3 (split 72.1; causal 73.4 and 69.6).
int32_t dq_splits(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H)
{
    const int64_t groups = B * H * ((Lq + kHeld - 1) / kHeld);
    const int64_t least = dt == IM2WIN_F32 ? 128 : 256, enough = groups < 256 ? 2 * least : 8 * least;
    if (groups <= 0 || groups >= 512 || Lk < enough)
        return 1;
    const int64_t s = (512 + groups - 1) / groups;
    return (int32_t)(s < Lk / least ? s : Lk / least);
}

// Floats of the partial strip gradients: one strip for each of attn_dq's
// workgroups.  R here is what is left of the range (attn_range).
int64_t strip_part_floats(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t R)
{
    const int64_t n = dq_splits(dt, B, Lq, Lk, H) * ((Lq + kHeld - 1) / kHeld);
    return R ? (B * H * n * (2 * R + 1) + 3) / 4 * 4 : 0;
}
int64_t dq_part_floats(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t D)
{
    const int64_t s = dq_splits(dt, B, Lq, Lk, H);
    return s > 1 ? s * B * H * Lq * D : 0;
}

// Workgroups that share the queries of one key tile: with few key/value heads
// and short rows there are fewer key tiles than the 256 CUs can work on, and
// causal masks need about two of them a CU to even out.  Measured, whole
// backward calls, one workgroup against split: bf16, 8 heads of 128 over 2,
// 2048 tokens 306 -> 118 us, 16 over 4, causal 345 -> 144; fp32, 3x6 heads of
// 80, 1001 tokens 426 -> 353.  With 256 key tiles the second one a CU pays
// under causal masks of long rows: 16 heads of 64, 2048 tokens 101 -> 102,
// causal 102 -> 92, but 2x16 heads, 1024 tokens 65 -> 73, causal 71 -> 73.  Four
// tiles each: fp16, 8 heads of 64, 512 tokens 35.8 (one each 40.5, two 35.7);
// short fp32 rows would take fewer: 4 heads of 64, 256 tokens 67 (46, 53).
int32_t dkdv_splits(int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv)
{
    const int64_t groups = B * Hkv * ((Lk + kHeld - 1) / kHeld), work = (H / Hkv) * ((Lq + 63) / 64);
    if (groups <= 0 || groups >= 512)
        return 1;
    int64_t s = (512 + groups - 1) / groups;
    if (s > work / 4)  // at least four tiles each
        s = work / 4;
    return s < 1 ? 1 : (int32_t)s;
}

int64_t dkdv_part_floats(int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D)
{
    const int64_t s = dkdv_splits(B, Lq, Lk, H, Hkv);
    return s > 1 ? s * B * Hkv * Lk * 2 * D : 0;
}

// Floats of attn_dq's strip and its gradients in LDS (even: 8-byte words follow).
__host__ __device__ inline int strip_floats(int R, int want_strip)
{
    return R ? ((2 * R + 1) * (want_strip ? 1 + 2 * kWaves : 1) + 1) / 2 * 2 : 0;
}

template <class Op>
constexpr float p_shift() { return 0.0f; }
template <>
constexpr float p_shift<F16Op>() { return 14.0f; }

constexpr int kStatRows = 64;  // rows a workgroup of row_stats, 16 lanes each
static_assert(kStatRows == kDocTile, "norm_tiles counts document ranges too");

// fp16: the largest |dout_i| and |v_j| that each workgroup of row_stats met,
// [B*Hkv][G*query tiles + key tiles].
__host__ __device__ inline int norm_tiles(int L) { return (L + kStatRows - 1) / kStatRows; }
__host__ __device__ inline int64_t norm_step(int G, int Lq, int Lk) { return (int64_t)G * norm_tiles(Lq) + norm_tiles(Lk); }

// The power of two that dS of a head group is multiplied by.
template <class Op>
__device__ inline float ds_scale(const AttnArgs &a, int b, int hk)
{
    if constexpr (sizeof(typename Op::elem) == 2 && p_shift<Op>() > 0) {
        const int nq = a.G * norm_tiles(a.Lq), nk = norm_tiles(a.Lk);
        const float *const p = a.norms + ((int64_t)b * a.Hkv + hk) * (nq + nk);
        float q = 0, v = 0;
        for (int i = threadIdx.x & 63; i < nq; i += 64)
            q = fmaxf(q, p[i]);
        for (int i = threadIdx.x & 63; i < nk; i += 64)
            v = fmaxf(v, p[nq + i]);
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) {
            q = fmaxf(q, __shfl_xor(q, m));
            v = fmaxf(v, __shfl_xor(v, m));
        }
        const float bound = 2.0f * q * v;
        const float e = bound > 0 ? floorf(15.0f - __log2f(bound) - 0.01f) : 0.0f;
        return exp2f(fminf(fmaxf(e, -40.0f), 40.0f));
    }
    return 1.0f;
}

// ---- row statistics ----

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

// *to = the largest of v over the workgroup.
__device__ inline void store_max(float *to, float v)
{
    __shared__ float w[kWaves];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        v = fmaxf(v, __shfl_xor(v, m));
    if ((threadIdx.x & 63) == 0)
        w[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        *to = fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3]));
}

// Whether some query sees key j; the 16 lanes of a group ask together.  With
// documents the queries are searched from the key's own position on, a tile of
// them a lane, where rows of packed documents find theirs at once.
__device__ inline bool seen_key(const AttnArgs &a, int b, int n, int j)
{
    const int off = first_pos(a, n);
    const int first = a.causal && !(a.prefix && j < a.prefix[b]) ? max(j - off, 0) : 0;
    if (j >= n || first >= a.Lq)
        return false;
    if (!a.k_doc)
        return true;
    const int doc = a.k_doc[(int64_t)b * a.Lk + j], tiles = norm_tiles(a.Lq), t0 = first / kDocTile, span = tiles - t0;
    const DocRange *const ranges = a.q_range + (int64_t)b * tiles;
    const int32_t *const ids = a.q_doc + (int64_t)b * a.Lq;
    const int begin = min(max(j - off, first) / kDocTile, tiles - 1);
    bool found = false;
    for (int s = threadIdx.x & 15; doc >= 0 && s < span && !found; s += 16) {
        const int t = begin + s < tiles ? begin + s : begin + s - span;
        const DocRange r = ranges[t];
        if (doc < r.lo || doc > r.hi)
            continue;
        found = !r.mixed;
        for (int i = max(t * kDocTile, first); i < min((t + 1) * kDocTile, a.Lq) && !found; ++i)
            found = ids[i] == doc;
    }
    return __ballot(found) >> (threadIdx.x & 48) & 0xffff;
}

// {lse*log2(e) - p_shift, dout.out} and, fp16, the largest |dout| (finite ones
// of queries that see something); the workgroups after those of the queries
// take, fp16, the largest |v| of the keys that a query sees.
template <class Op>
__global__ __launch_bounds__(kThreads) void row_stats(AttnArgs a)
{
    const int d = (threadIdx.x & 15) * 8, tq = norm_tiles(a.Lq), tk = norm_tiles(a.Lk);
    const uint32_t queries = (uint32_t)(a.B * a.H) * tq;
    float most = 0;
    if (blockIdx.x >= queries) {
        const uint32_t id = blockIdx.x - queries, kv = id / tk;
        const int t = id - kv * tk, b = kv / a.Hkv, hk = kv - b * a.Hkv, n = keys_of(a, b);
#pragma unroll
        for (int k = 0; k < kStatRows / 16; ++k) {
            const int j = t * kStatRows + k * 16 + (threadIdx.x >> 4);
            float f[8], sq = 0;
            if (seen_key(a, b, n, j) && d < a.D) {
                load8<Op>(a.v + b * a.v_sb + hk * a.v_sh + (int64_t)j * a.v_st + d * sizeof(typename Op::elem), f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sq += f[e] * f[e];
            }
            sq = sum16(sq);
            most = fmaxf(most, sq < INFINITY ? sq : 0.0f);
        }
        store_max(a.norms + kv * norm_step(a.G, a.Lq, a.Lk) + a.G * tq + t, sqrtf(most));
        return;
    }
    const uint32_t bh = blockIdx.x / tq;
    const int t = blockIdx.x - bh * tq, b = bh / a.H, hq = bh - b * a.H;
    const int Lp = stat_rows(a.Lq);
    float *const stat = a.stat + (int64_t)bh * 2 * Lp;
#pragma unroll
    for (int k = 0; k < kStatRows / 16; ++k) {
        const int i = t * kStatRows + k * 16 + (threadIdx.x >> 4);
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
        const float l = i < a.Lq ? a.lse[(int64_t)bh * a.Lq + i] : -INFINITY;
        const bool some = l != -INFINITY;
        if (d == 0) {
            stat[i] = some ? l * kLog2e - p_shift<Op>() : INFINITY;
            stat[Lp + i] = i < a.Lq ? dot : 0.0f;
        }
        if constexpr (p_shift<Op>() > 0) {
            sq = sum16(sq);
            most = fmaxf(most, some && sq < INFINITY ? sq : 0.0f);
        }
    }
    if constexpr (p_shift<Op>() > 0)
        store_max(a.norms + ((int64_t)b * a.Hkv + hq / a.G) * norm_step(a.G, a.Lq, a.Lk) + hq % a.G * tq + t, sqrtf(most));
}

// ---- what both kernels do with a 32 x 32 tile of scores ----

// Exponents of the probabilities (base 2), without the bias: the scores of
// the products in s less lse(r), the row statistic of register r; slope:
// 1 - tanh^2 where scores are capped, a quarter of it in kCapped instances
// (slope_scale has the rest).  Those round P and dS to 16 bits and give
// nothing else, so they take tanh(u) = 1 - 2*r, r = 1/(1 + e^2u), in four
// operations.  Its error of 1.2e-7 whatever u is becomes one of 1.2e-7*cap in
// the exponent, and so in P: up to kCappedMost 3.1e-5 at most, a sixteenth of
// fp16's rounding of P (2^-11) and a 128th of bf16's.  Larger caps go to the
// kAny instances, whose series for small u is exact to fp32.
constexpr float kCappedMost = 256.0f;
template <int FEAT>
__device__ constexpr float slope_scale() { return FEAT == kCapped ? 4.0f : 1.0f; }
template <int FEAT, class Lse>
__device__ inline void to_scores(f32x16_acc &s, f32x16_acc &slope, const ScoreArgs &c, Lse lse)
{
    if constexpr (FEAT == kCapped) {
        const float c1 = c.c1 * (2.0f * kLog2e);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float t = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s[r] * c1));
            slope[r] = fmaf(-t, t, t);
            s[r] = fmaf(-2.0f * c.c2, t, c.c2 - lse(r));
        }
    } else if (FEAT == kAny && c.cap) {
        f32x16_acc t[1] = {s};
        tanh_scores(t, c.c1);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            slope[r] = fmaf(-t[0][r], t[0][r], 1.0f);
            s[r] = fmaf(c.c2, t[0][r], -lse(r));
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[r] = fmaf(s[r], c.c1, -lse(r));
    }
}

template <class Op, int DP>
struct Bwd {
    typedef Tile<Op, DP> T;
    static constexpr int kRows = OpInfo<Op>::kIs32 ? 32 : 64;  // streamed tokens a tile
    static constexpr int kSub = kRows / 32;
    static constexpr int kTileBytes = kRows * T::kRowBytes;
    // waves a SIMD to fit in, and whether the dk/dv kernel, alone on its SIMD
    // with more than 256 registers, reads fragments ahead
    static constexpr int kOccKV = T::kRowBytes <= 128 ? 2 : 1, kOccQ = T::kRowBytes <= 256 ? 2 : 1;
    static constexpr bool kAhead = kOccKV == 1 && !OpInfo<Op>::kIs32;
};

// ---- dk, dv: a key per lane ----
template <class Op, int DP, int FEAT>
__global__ __launch_bounds__(kThreads, (Bwd<Op, DP>::kOccKV)) void attn_dkdv(AttnArgs a)
{
    typedef Bwd<Op, DP> W;
    typedef Tile<Op, DP> T;
    typedef typename Op::v8 V8;
    // two slots of a tile of q and dout, and of their rows' statistics; each
    // an array of its own: the compiler can tell that reading one does not
    // wait for the loads that land in the other
    __shared__ __align__(16) char slot0[2 * W::kTileBytes];
    __shared__ __align__(16) char slot1[2 * W::kTileBytes];
    __shared__ __align__(16) float rows0[192];  // 64 of lse, delta, documents
    __shared__ __align__(16) float rows1[192];
    __shared__ int shared_first[kWaves], shared_lo[kWaves], shared_hi[kWaves];
    extern __shared__ __align__(16) float strip[];  // 2R+1, times log2(e); documents: a bit for each query tile

    // `splits` workgroups share the (head, query tile) pairs of a key tile
    const Work work = work_item(a.B * a.Hkv, a.splits, a.tiles, a.causal, blockIdx.x);
    const int kt = work.tile, b = work.kv / a.Hkv, hk = work.kv - b * a.Hkv;  // early keys: long columns of causal masks
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
    const int t_first = __builtin_amdgcn_readfirstlane(wg_first) / W::kRows;
    const int tiles = (a.Lq + W::kRows - 1) / W::kRows;
    const DocRange *const ranges = a.k_doc ? a.q_range + (int64_t)b * ((a.Lq + kDocTile - 1) / kDocTile) : nullptr;
    uint64_t *const bits = (uint64_t *)(strip + (a.R ? 2 * a.R + 2 : 0));
    if (a.k_doc) {
        mark_tiles(bits, ranges, tiles, W::kRows, wg_lo, wg_hi, wave, lane);
        __syncthreads();
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
    const float f = dss * exp2f(-p_shift<Op>());  // dS*dss = P' * f*(dP - delta)
    const int Lp = stat_rows(a.Lq);

    // this workgroup's pairs u of head u / span and tile t_first + u % span
    const int span = max(tiles - t_first, 0);
    const int u_end = (int)((int64_t)span * a.G * (work.g + 1) / a.splits);
    for (int u = (int)((int64_t)span * a.G * work.g / a.splits); u < u_end;) {
        const int g = u / span, hq = hk * a.G + g;
        const int t_begin = t_first + (u - g * span), t_end = min(tiles, t_begin + (u_end - u));
        u += t_end - t_begin;
        const char *const qp = a.q + b * a.q_sb + hq * a.q_sh, *const dop = a.dout + b * a.do_sb + hq * a.do_sh;
        const float *const stat = a.stat + ((int64_t)b * a.H + hq) * 2 * Lp;
        auto issue = [&](char *slot, float *rows, int t) {
            const int q0 = t * W::kRows;
            T::template dma<W::kRows, kWaves>(slot, qp + (int64_t)q0 * a.q_st, a.q_st, a.Lq - q0, a.D, wave, lane);
            T::template dma<W::kRows, kWaves>(slot + W::kTileBytes, dop + (int64_t)q0 * a.do_st, a.do_st, a.Lq - q0, a.D,
                                              wave, lane);
            if (wave < 2)  // statistics have whole tiles of rows
                dma_words(rows + 64 * wave, stat + wave * Lp + q0, W::kRows, lane);
            else if (wave == 2 && a.k_doc)
                dma_words(rows + 128, a.q_doc + (int64_t)b * a.Lq + q0, a.Lq - q0, lane);
        };
        auto after = [&](int t) { return a.k_doc ? next_tile(bits, t, t_end) : t; };
        auto step = [&](char *slot, float *rows, char *other, float *other_rows, int x) {
            wait_loads<0>();
            ring_barrier();
            const int next = after(x + 1), q0 = x * W::kRows;
            if (next < t_end)
                issue(other, other_rows, next);
            DocRange dr = {0, 0, 0, 0};
            if (a.k_doc)
                dr = ranges[q0 / kDocTile];
            if (q0 + W::kRows <= least || (a.k_doc && !(dr.lo <= dhi && dr.hi >= dlo)))
                return next;
            const bool docs_differ = a.k_doc && (dr.mixed || dlo != dhi || dr.lo != dlo);
            const bool partial = q0 < most || docs_differ;
            const char *const tq = slot, *const tdo = slot + W::kTileBytes;
            const uint32_t roff = opaque(T::row_offset(lane)), coff = opaque(T::col_offset(lane));
            // products of 32 rows and this wave's keys: s = q k, dp = dout v
            auto scores = [&](int t, f32x16_acc &s, f32x16_acc &dp) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = dp[r] = 0;
                V8 buf[2][4];  // two steps of 16 channels, q and dout
                auto load = [&](int i, V8(&c)[4]) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        c[2 * x] = T::row_frag(tq, roff, t, 2 * i + x);
                        c[2 * x + 1] = T::row_frag(tdo, roff, t, 2 * i + x);
                    }
                };
                if constexpr (W::kAhead)
                    load(0, buf[0]);
                pipeline<Op, W::kAhead, DP / 32, 4>(buf, load, [&](int i, const V8(&c)[4]) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        s = Op::mfma(c[2 * x], kf[2 * i + x], s);
                        dp = Op::mfma(c[2 * x + 1], vf[2 * i + x], dp);
                    }
                });
            };
            // their probabilities and score gradients, in place
            auto gradients = [&](int t, f32x16_acc &s, f32x16_acc &dp) {
                const float *const lse = rows + 32 * t + 4 * h, *const delta = lse + 64;  // of row reg_row(r)
                f32x16_acc slope;
                to_scores<FEAT>(s, slope, sc, [&](int r) { return lse[reg_row(r)]; });
                const int i0 = q0 + 32 * t;
                if (FEAT == kAny && a.R) {
                    const int dmin = jlo - (i0 + 31 + off), dmax = jhi - (i0 + off);
                    if (dmax <= -a.R || dmin >= a.R) {
                        const float far = strip[dmin >= a.R ? 2 * a.R : 0];
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            s[r] += far;
                    } else if (dmin >= -a.R && dmax <= a.R) {
                        const float *const at = strip + (j - (i0 + 4 * h + off) + a.R);
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            s[r] += at[-reg_row(r)];
                    } else {
                        const int d0 = j - (i0 + 4 * h + off);
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            s[r] += strip[min(max(d0 - reg_row(r), -a.R), a.R) + a.R];
                    }
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = __builtin_amdgcn_exp2f(s[r]);
                    float d = dp[r] - delta[reg_row(r)];
                    if constexpr (p_shift<Op>() > 0)
                        d *= f;
                    dp[r] = s[r] * d;
                }
                if (FEAT == kAny ? sc.cap : FEAT == kCapped)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        dp[r] *= slope[r];
            };
            // dv += dout^T p, dk += q^T ds: 16 rows and 32 channels a step
            constexpr int N = DP / 32;
            auto columns = [&](int t, int i, V8(&c)[2]) {
                c[0] = T::col_frag(tdo, coff, 32 * t + 16 * (i / N), i % N);
                c[1] = T::col_frag(tq, coff, 32 * t + 16 * (i / N), i % N);
            };
            uint32_t bad_dout = 0, bad_q = 0;  // fragments of dout and q had values that are not finite
            auto sums = [&](int t, const V8(&p)[2], const V8(&ds)[2], V8(&buf)[2][2], auto each) {
                pipeline<Op, W::kAhead, 2 * N, 2>(
                    buf, [&](int i, V8(&c)[2]) { columns(t, i, c); },
                    [&](int i, const V8(&c)[2]) {
                        dv[i % N] = Op::mfma(each(c[0], bad_dout), p[i / N], dv[i % N]);
                        dk[i % N] = Op::mfma(each(c[1], bad_q), ds[i / N], dk[i % N]);
                    });
            };
            auto same = [](V8 c, uint32_t &) { return c; };
#pragma unroll
            for (int t = 0; t < W::kSub; ++t) {
                f32x16_acc s, dp;
                V8 p[2], ds[2], cbuf[2][2];
                scores(t, s, dp);
                if constexpr (W::kAhead) {  // these travel while the exponentials are taken
                    columns(t, 0, cbuf[0]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                gradients(t, s, dp);
                if (q0 + 32 * t + 32 > a.Lq) {
                    // rows past Lq hold zeros, which times a key or value
                    // that is infinite or NaN are not zero
                    const int end = a.Lq - (q0 + 32 * t) - 4 * h;
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        s[r] = reg_row(r) < end ? s[r] : 0.0f;
                        dp[r] = reg_row(r) < end ? dp[r] : 0.0f;
                    }
                }
                if (partial) {
                    const int lim = first == INT32_MAX ? INT32_MAX : first - (q0 + 32 * t) - 4 * h;
                    const float *const at = rows + 32 * t + 4 * h;  // + 128: document
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const bool out =
                            reg_row(r) < lim || (docs_differ && __float_as_int(at[128 + reg_row(r)]) != doc);
                        s[r] = out ? 0.0f : s[r];
                        dp[r] = out ? 0.0f : dp[r];
                    }
                }
                // rounded to 16 bits as operands of the matrix cores, whose
                // fp32 products cost 7 times as much (154 against 1121
                // TFLOP/s); all sums of them are fp32
                pack16<Op>(s, p);
                pack16<Op>(dp, ds);
                if (partial) {
                    // a left-out pair's zero times infinity or NaN must stay zero
                    bad_dout = 0;
                    sums(t, p, ds, cbuf, [](V8 c, uint32_t &bad) { return finite<Op>(c, bad); });
                    if (__any(bad_dout)) {
                        // rows of dout that are not finite reach the keys they
                        // see (those of q do through ds, which is NaN)
                        for (int rr = 0; rr < 32; ++rr) {
                            if (q0 + 32 * t + rr < first ||
                                (docs_differ && __float_as_int(rows[128 + 32 * t + rr]) != doc))
                                continue;
#pragma unroll
                            for (int dt = 0; dt < N; ++dt)
#pragma unroll
                                for (int g4 = 0; g4 < 4; ++g4) {
                                    float v[4];
                                    T::four(tdo, 32 * t + rr, 32 * dt + 8 * g4 + 4 * h, v);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        dv[dt][4 * g4 + e] += fabsf(v[e]) < INFINITY ? 0.0f : v[e];
                                }
                        }
                    }
                } else {
                    sums(t, p, ds, cbuf, same);
                }
            }
            return next;
        };
        __syncthreads();  // the head before this one has read its tiles and strip
        int t = after(t_begin);
        if (t < t_end)
            issue(slot0, rows0, t);
        if (FEAT == kAny && a.R) {
            for (int x = threadIdx.x; x < 2 * a.R + 1; x += kThreads)
                strip[x] = a.strip[hq * a.strip_step + x] * kLog2e;
            ring_barrier();
        }
        while (t < t_end) {
            t = step(slot0, rows0, slot1, rows1, t);
            if (t >= t_end)
                break;
            t = step(slot1, rows1, slot0, rows0, t);
        }
    }
    if (!in)
        return;
    if (a.splits > 1) {  // sums as they are; dkdv_join adds the splits
        float *const part = a.part + (((int64_t)work.g * a.B * a.Hkv + work.kv) * a.Lk + j) * 2 * a.D;
        store_row<F32Op, DP>((char *)part, dk, slope_scale<FEAT>() * a.scale / dss, h, a.D);
        store_row<F32Op, DP>((char *)(part + a.D), dv, exp2f(-p_shift<Op>()), h, a.D);
        return;
    }
    store_row<Op, DP>(a.dk + b * a.dk_sb + hk * a.dk_sh + (int64_t)j * a.dk_st, dk, slope_scale<FEAT>() * a.scale / dss, h, a.D);
    store_row<Op, DP>(a.dv + b * a.dv_sb + hk * a.dv_sh + (int64_t)j * a.dv_st, dv, exp2f(-p_shift<Op>()), h, a.D);
}

// ---- dq (and the strip's gradient): a query per lane ----

// Sums of a 32x32 tile along its diagonals.  Lane i of 16 (one query each)
// holds rows k = reg_row(r) (the lane half's 4*h apart), on diagonal k - i.
// Moving row k = 16*c + n down by n lanes puts diagonal 16*c - i into lane i,
// and what leaves the 16 lanes at the bottom re-enters at the top on diagonal
// 16*(c+1) - i: two adds an element whose operand moves on the way.
// sum[x] of lane i: diagonal 16*x - i.
template <int N>
__device__ inline void move_add(float v, float &here, float &next)
{
    if constexpr (N == 0) {
        here += v;
    } else {
        // row_shl:N and row_shr:(16-N); lanes without a source take 0
        here += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x100 + N, 0xf, 0xf, true));
        next += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x110 + 16 - N, 0xf, 0xf, true));
    }
}

__device__ inline void diagonal_sums(const f32x16_acc &v, f32x4_acc &sum)
{
    float a = 0, b = 0, c = 0;
    move_add<0>(v[0], a, b);
    move_add<1>(v[1], a, b);
    move_add<2>(v[2], a, b);
    move_add<3>(v[3], a, b);
    move_add<8>(v[4], a, b);
    move_add<9>(v[5], a, b);
    move_add<10>(v[6], a, b);
    move_add<11>(v[7], a, b);
    move_add<0>(v[8], b, c);
    move_add<1>(v[9], b, c);
    move_add<2>(v[10], b, c);
    move_add<3>(v[11], b, c);
    move_add<8>(v[12], b, c);
    move_add<9>(v[13], b, c);
    move_add<10>(v[14], b, c);
    move_add<11>(v[15], b, c);
    sum[0] = a;
    sum[1] = b;
    sum[2] = c;
}

template <class Op, int DP, int FEAT>
__global__ __launch_bounds__(kThreads, (Bwd<Op, DP>::kOccQ)) void attn_dq(AttnArgs a, int want_strip)
{
    typedef Bwd<Op, DP> W;
    typedef Tile<Op, DP> T;
    typedef typename Op::v8 V8;
    __shared__ __align__(16) char slot0[2 * W::kTileBytes];
    __shared__ __align__(16) char slot1[2 * W::kTileBytes];
    __shared__ int kdoc0[64], kdoc1[64];
    // [1 or 1 + 2*kWaves][2R+1]: the strip times log2(e), its gradients; documents: a bit for each key tile
    extern __shared__ __align__(16) float strip[];
    const int width = 2 * a.R + 1;
    __shared__ int shared_most[kWaves], shared_lo[kWaves], shared_hi[kWaves];

    // `splits` workgroups share the keys of a query tile
    const Work work = work_item(a.B * a.Hkv, a.G * a.splits, a.tiles, a.causal, blockIdx.x);
    const int qt = a.tiles - 1 - work.tile;  // long rows of causal masks first
    const int split = work.g / a.G;
    const int b = work.kv / a.Hkv, hk = work.kv - b * a.Hkv, hq = hk * a.G + work.g % a.G;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = qt * kHeld + wave * 32 + (lane & 31);
    const bool live = i < a.Lq;
    const int n = keys_of(a, b);
    const int pos = i + first_pos(a, n);
    int lim = n, doc = -1;
    if (a.causal)
        lim = max(0, min(n, max(pos + 1, a.prefix ? a.prefix[b] : 0)));
    if (a.q_doc) {
        if (live)
            doc = a.q_doc[(int64_t)b * a.Lq + i];
        if (doc < 0)
            lim = 0;
    }
    // A lane without a query holds zeros and an lse of infinity.  Its column
    // of dq is not stored; of the strip's gradient, which is summed over
    // lanes, it is left out: zero times a key or value that is infinite or NaN
    // is not zero.
    const bool some_dead = qt * kHeld + wave * 32 + 32 > a.Lq;
    const int most = wave_max(live ? lim : 0), least = wave_min(live ? lim : INT32_MAX);
    const int plo = wave_min(pos), phi = wave_max(pos);
    const bool seen = live && lim > 0;
    const int dlo = wave_min(seen ? doc : INT32_MAX), dhi = wave_max(seen ? doc : -1);
    // each half wave has a strip of gradients of its own, to which it adds by
    // LDS atomics: the 32 lanes that add in one instruction hold 32 different
    // distances, and no other wave adds, so nothing is summed in an order that
    // could change
    float *const grad = strip + width * (1 + 2 * wave + h);
    float far_lo = 0, far_hi = 0;
    if (FEAT == kAny && a.R)
        for (int t = threadIdx.x; t < width; t += kThreads) {
            strip[t] = a.strip[hq * a.strip_step + t] * kLog2e;
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
    const int Lp = stat_rows(a.Lq);
    const float *const stat = a.stat + ((int64_t)b * a.H + hq) * 2 * Lp;
    const float lse = live ? stat[i] : INFINITY, row_delta = live ? stat[Lp + i] : 0.0f;
    const float dss = ds_scale<Op>(a, b, hk);
    const float delta = row_delta * dss * exp2f(-p_shift<Op>());
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

    const int all_tiles = (__builtin_amdgcn_readfirstlane(wg_most) + W::kRows - 1) / W::kRows;
    const int tiles = (int)((int64_t)all_tiles * (split + 1) / a.splits);  // the first tile not this workgroup's
    const DocRange *const ranges = a.q_doc ? a.k_range + (int64_t)b * ((a.Lk + kDocTile - 1) / kDocTile) : nullptr;
    uint64_t *const bits = (uint64_t *)(strip + strip_floats(a.R, want_strip));
    if (a.q_doc) {
        mark_tiles(bits, ranges, tiles, W::kRows, wg_lo, wg_hi, wave, lane);
        __syncthreads();
    }
    auto issue = [&](char *slot, int *ids, int t) {
        const int k0 = t * W::kRows;
        T::template dma<W::kRows, kWaves>(slot, kp + (int64_t)k0 * a.k_st, a.k_st, n - k0, a.D, wave, lane);
        T::template dma<W::kRows, kWaves>(slot + W::kTileBytes, vp + (int64_t)k0 * a.v_st, a.v_st, n - k0, a.D, wave,
                                          lane);
        if (a.q_doc && wave == 0)
            dma_words(ids, a.k_doc + (int64_t)b * a.Lk + k0, n - k0, lane);
    };
    auto after = [&](int t) { return a.q_doc ? next_tile(bits, t, tiles) : t; };
    auto step = [&](char *slot, int *kdoc, char *other, int *other_ids, int at) {
        wait_loads<0>();
        ring_barrier();
        const int next = after(at + 1), k0 = at * W::kRows;
        if (next < tiles)
            issue(other, other_ids, next);
        DocRange dr = {0, 0, 0, 0};
        if (a.q_doc)
            dr = ranges[k0 / kDocTile];
        const char *const tk = slot, *const tv = slot + W::kTileBytes;
        const uint32_t roff = opaque(T::row_offset(lane)), coff = opaque(T::col_offset(lane));
        if (k0 >= most || (a.q_doc && !(dr.lo <= dhi && dr.hi >= dlo)))
            return next;
        const bool docs_differ = a.q_doc && (dr.mixed || dlo != dhi || dr.lo != dlo);
        const bool partial = k0 + W::kRows > least || docs_differ;
#pragma unroll
        for (int t = 0; t < W::kSub; ++t) {
            f32x16_acc s, dp, slope;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[r] = dp[r] = 0;
            {
                V8 buf[2][4];  // two steps of 16 channels, k and v
                auto load = [&](int i, V8(&c)[4]) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        c[2 * x] = T::row_frag(tk, roff, t, 2 * i + x);
                        c[2 * x + 1] = T::row_frag(tv, roff, t, 2 * i + x);
                    }
                };
                pipeline<Op, false, DP / 32, 4>(buf, load, [&](int i, const V8(&c)[4]) {
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        s = Op::mfma(c[2 * x], qf[2 * i + x], s);
                        dp = Op::mfma(c[2 * x + 1], dof[2 * i + x], dp);
                    }
                });
            }
            V8 cbuf[2][DP / 32];  // 16 keys, all channels
            auto cload = [&](int i, V8(&c)[DP / 32]) {
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt)
                    c[dt] = T::col_frag(tk, coff, 32 * t + 16 * i, dt);
            };
            to_scores<FEAT>(s, slope, sc, [&](int) { return lse; });
            const int j0 = k0 + 32 * t, d0 = j0 + 4 * h - pos;
            const bool far = FEAT == kAny && a.R && (j0 + 31 - plo <= -a.R || j0 - phi >= a.R);
            if (FEAT == kAny && a.R) {
                if (far) {
                    const float v = strip[j0 - phi >= a.R ? 2 * a.R : 0];
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] += v;
                } else if (j0 - phi >= -a.R && j0 + 31 - plo <= a.R) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] += strip[d0 + a.R + reg_row(r)];
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[r] += strip[min(max(d0 + reg_row(r), -a.R), a.R) + a.R];
                }
            }
            const int last = lim - j0 - 4 * h;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(s[r]);
                float ds = p * fmaf(dp[r], f, -delta);
                if (partial)
                    ds = reg_row(r) >= last || (docs_differ && kdoc[32 * t + reg_row(r) + 4 * h] != doc) ? 0.0f : ds;
                dp[r] = ds;
            }
            if (FEAT == kAny && want_strip) {
                if (some_dead)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        dp[r] = live ? dp[r] : 0.0f;
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
                    f32x4_acc sum;
                    diagonal_sums(dp, sum);
#pragma unroll
                    for (int x = 0; x < 3; ++x) {
                        const int d = j0 + 4 * h + 16 * x - pos;
                        far_lo += d <= -a.R ? sum[x] : 0.0f;
                        far_hi += d >= a.R ? sum[x] : 0.0f;
                        if (d > -a.R && d < a.R)
                            __hip_atomic_fetch_add(grad + d + a.R, sum[x], __ATOMIC_RELAXED,
                                                   __HIP_MEMORY_SCOPE_WAVEFRONT);
                    }
                }
            }
            if (FEAT == kAny ? sc.cap : FEAT == kCapped) {
                if (partial) {
                    // the slope of a left-out score may be NaN
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        dp[r] = dp[r] == 0.0f ? 0.0f : dp[r] * slope[r];
                } else {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        dp[r] *= slope[r];
                }
            }
            if (!partial) {
                pipeline<Op, false, 2, DP / 32>(cbuf, cload, [&](int i, const V8(&c)[DP / 32]) {
                    const V8 ds = pack8<Op>(dp, 8 * i);
#pragma unroll
                    for (int dt = 0; dt < DP / 32; ++dt)
                        dq[dt] = Op::mfma(c[dt], ds, dq[dt]);
                });
                continue;
            }
            uint32_t bad = 0;
            pipeline<Op, false, 2, DP / 32>(cbuf, cload, [&](int i, const V8(&c)[DP / 32]) {
                const V8 ds = pack8<Op>(dp, 8 * i);
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt)
                    dq[dt] = Op::mfma(finite<Op>(c[dt], bad), ds, dq[dt]);
            });
        }
        return next;
    };
    int t = after((int)((int64_t)all_tiles * split / a.splits));
    if (t < tiles)
        issue(slot0, kdoc0, t);
    while (t < tiles) {
        t = step(slot0, kdoc0, slot1, kdoc1, t);
        if (t >= tiles)
            break;
        t = step(slot1, kdoc1, slot0, kdoc0, t);
    }
    if (live && a.splits > 1)  // sums as they are; dq_join adds the splits
        store_row<F32Op, DP>((char *)(a.part + (((int64_t)split * a.B * a.H + (int64_t)b * a.H + hq) * a.Lq + i) * a.D), dq,
                             slope_scale<FEAT>() * a.scale / dss, h, a.D);
    else if (live)
        store_row<Op, DP>(a.dq + b * a.dq_sb + hq * a.dq_sh + (int64_t)i * a.dq_st, dq, slope_scale<FEAT>() * a.scale / dss, h, a.D);
    if (FEAT != kAny || !want_strip)
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
    float *out = a.strip_part + ((((int64_t)hq * a.B + b) * a.splits + split) * a.tiles + qt) * width;
    for (int t = threadIdx.x; t < width; t += kThreads) {
        float v = 0;
#pragma unroll
        for (int w = 1; w <= 2 * kWaves; ++w)
            v += strip[w * width + t];
        out[t] = v / dss;
    }
}

// dk and dv of a key: the sum of the splits, four channels a lane.
template <class Op>
__global__ __launch_bounds__(kThreads) void dkdv_join(AttnArgs a)
{
    const int per = a.D / 2;  // lanes a key
    const int64_t keys = (int64_t)a.B * a.Hkv * a.Lk, id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t key = id / per;
    if (key >= keys)
        return;
    const int d = (int)(id - key * per) * 4;
    typedef float v4 __attribute__((ext_vector_type(4)));
    v4 v = {0, 0, 0, 0};
    for (int s = 0; s < a.splits; ++s)
        v += *(const v4 *)(a.part + (s * keys + key) * 2 * a.D + d);
    const int64_t kv = key / a.Lk, j = key - kv * a.Lk, b = kv / a.Hkv, hk = kv - b * a.Hkv;
    char *const p = d < a.D ? a.dk + b * a.dk_sb + hk * a.dk_sh + j * a.dk_st : a.dv + b * a.dv_sb + hk * a.dv_sh + j * a.dv_st;
    typedef typename Op::elem V __attribute__((ext_vector_type(4)));
    V o;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        o[e] = (typename Op::elem)v[e];
    *(V *)(p + (d < a.D ? d : d - a.D) * sizeof(typename Op::elem)) = o;
}

// dq of a query: the sum of the splits, four channels a lane.
template <class Op>
__global__ __launch_bounds__(kThreads) void dq_join(AttnArgs a)
{
    const int per = a.D / 4;  // lanes a query
    const int64_t rows = (int64_t)a.B * a.H * a.Lq, id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t row = id / per;
    if (row >= rows)
        return;
    const int d = (int)(id - row * per) * 4;
    typedef float v4 __attribute__((ext_vector_type(4)));
    v4 v = {0, 0, 0, 0};
    for (int s = 0; s < a.splits; ++s)
        v += *(const v4 *)(a.part + (s * rows + row) * a.D + d);
    const int64_t bh = row / a.Lq, i = row - bh * a.Lq, b = bh / a.H, hq = bh - b * a.H;
    typedef typename Op::elem V __attribute__((ext_vector_type(4)));
    V o;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        o[e] = (typename Op::elem)v[e];
    *(V *)(a.dq + b * a.dq_sb + hq * a.dq_sh + i * a.dq_st + d * sizeof(typename Op::elem)) = o;
}

// dstrip[h][x]: the sum of `n` partial strips, which hold the `width` middle
// entries of the `full` that a strip has (the others have no pair), 64 entries
// a workgroup, each by 16 lanes that take every 16th strip.  A grid has at
// most kMaxGridY heads; its workgroups take more in turn.
constexpr int kReducers = 16;
constexpr int kMaxGridY = 65535;
__global__ __launch_bounds__(64 * kReducers) void strip_reduce(const float *__restrict__ part,
                                                               float *__restrict__ dstrip, int32_t n, int32_t width,
                                                               int32_t full, int32_t H)
{
    __shared__ float s[kReducers][64];
    const int x = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
    const int c = x - (full - width) / 2;
    for (int h = blockIdx.y; h < H; h += gridDim.y) {
        float v = 0;
        if (c >= 0 && c < width)
#pragma unroll 4
            for (int r = k; r < n; r += kReducers)
                v += part[((int64_t)h * n + r) * width + c];
        s[k][threadIdx.x & 63] = v;
        __syncthreads();
        if (k == 0 && x < full) {
            v = 0;
#pragma unroll
            for (int r = 0; r < kReducers; ++r)
                v += s[r][threadIdx.x];
            dstrip[(int64_t)h * full + x] = v;
        }
        __syncthreads();
    }
}

template <class Op, int DP, int FEAT>
hipError_t run(const AttnArgs &a, float *dstrip, hipStream_t st)
{
    typedef Bwd<Op, DP> W;
    constexpr int dt = __is_same(Op, F32Op) ? IM2WIN_F32 : __is_same(Op, F16Op) ? IM2WIN_F16 : IM2WIN_BF16;
    const int width = 2 * a.R + 1;
    AttnArgs b = a;
    hipError_t e;
    const uint32_t stat_groups = (uint32_t)(a.B * a.H) * norm_tiles(a.Lq) +
                                 (p_shift<Op>() > 0 ? (uint32_t)(a.B * a.Hkv) * norm_tiles(a.Lk) : 0);
    if (stat_groups)
        row_stats<Op><<<stat_groups, kThreads, 0, st>>>(b);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;

    // LDS beside the tiles: strips and a bit for each streamed tile
    const size_t bits_k = a.q_doc ? (a.Lk + 64 * W::kRows - 1) / (64 * W::kRows) * 8 : 0;
    const size_t bits_q = a.q_doc ? (a.Lq + 64 * W::kRows - 1) / (64 * W::kRows) * 8 : 0;
    const size_t lds_kv = (a.R ? (2 * a.R + 2) * 4 : 0) + bits_q;
    const size_t lds_q = strip_floats(a.R, dstrip != nullptr) * 4 + bits_k;
    if (lds_kv && (e = hipFuncSetAttribute((const void *)attn_dkdv<Op, DP, FEAT>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                           16 << 10)) != hipSuccess)
        return e;
    if (lds_q && (e = hipFuncSetAttribute((const void *)attn_dq<Op, DP, FEAT>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                          84 << 10)) != hipSuccess)
        return e;
    b.tiles = (a.Lk + kHeld - 1) / kHeld;
    if (a.B * b.tiles) {
        b.splits = dkdv_splits(a.B, a.Lq, a.Lk, a.H, a.Hkv);
        attn_dkdv<Op, DP, FEAT><<<(uint32_t)(a.B * a.Hkv) * b.tiles * b.splits, kThreads, lds_kv, st>>>(b);
        const int64_t lanes = (int64_t)a.B * a.Hkv * a.Lk * (a.D / 2);
        if (b.splits > 1)
            dkdv_join<Op><<<(uint32_t)((lanes + kThreads - 1) / kThreads), kThreads, 0, st>>>(b);
    }
    b.tiles = (a.Lq + kHeld - 1) / kHeld;
    b.splits = dq_splits(dt, a.B, a.Lq, a.Lk, a.H);
    b.part = a.part + dkdv_part_floats(a.B, a.Lq, a.Lk, a.H, a.Hkv, a.D);
    b.strip_part = b.part + dq_part_floats(dt, a.B, a.Lq, a.Lk, a.H, a.D);
    if (a.B * b.tiles) {
        attn_dq<Op, DP, FEAT><<<(uint32_t)(a.B * a.H) * b.tiles * b.splits, kThreads, lds_q, st>>>(b, dstrip != nullptr);
        const int64_t lanes = (int64_t)a.B * a.H * a.Lq * (a.D / 4);
        if (b.splits > 1)
            dq_join<Op><<<(uint32_t)((lanes + kThreads - 1) / kThreads), kThreads, 0, st>>>(b);
    }
    if (dstrip) {
        const dim3 grid((uint32_t)((a.strip_step + 63) / 64), (uint32_t)(a.H < kMaxGridY ? a.H : kMaxGridY));
        strip_reduce<<<grid, 64 * kReducers, 0, st>>>(b.strip_part, dstrip, a.B * b.tiles * b.splits, width,
                                                      (int32_t)a.strip_step, a.H);
    }
    return hipGetLastError();
}

template <class Op, int DP>
hipError_t run_feat(const AttnArgs &a, float *dstrip, hipStream_t st)
{
    if constexpr (!OpInfo<Op>::kIs32) {
        if (!a.R && a.cap <= kCappedMost)
            return a.cap > 0 ? run<Op, DP, kCapped>(a, dstrip, st) : run<Op, DP, kPlain>(a, dstrip, st);
    }
    return run<Op, DP, kAny>(a, dstrip, st);
}

template <class Op>
hipError_t run_dim(const AttnArgs &a, float *dstrip, hipStream_t st)
{
    return a.D <= 32 ? run_feat<Op, 32>(a, dstrip, st)
         : a.D <= 64 ? run_feat<Op, 64>(a, dstrip, st)
         : a.D <= 96 ? run_feat<Op, 96>(a, dstrip, st)
                     : run_feat<Op, 128>(a, dstrip, st);
}

}  // namespace

int64_t attn_norm_bytes(int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv)
{
    return B * Hkv * norm_step((int)(H / Hkv), (int)Lq, (int)Lk) * 4;
}

int64_t attn_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D, int64_t R,
                        bool backward)
{
    if (!backward)
        return attn_forward_part_bytes(dt, B, Lq, Lk, H, Hkv, D);
    return (dkdv_part_floats(B, Lq, Lk, H, Hkv, D) + dq_part_floats(dt, B, Lq, Lk, H, D) +
            strip_part_floats(dt, B, Lq, Lk, H, attn_range(R, Lq, Lk))) * 4;
}

hipError_t launch_attn_backward(const AttnArgs &a, int dt, float *dstrip, hipStream_t st)
{
    return dt == IM2WIN_F32   ? run_dim<F32Op>(a, dstrip, st)
           : dt == IM2WIN_F16 ? run_dim<F16Op>(a, dstrip, st)
                              : run_dim<BF16Op>(a, dstrip, st);
}

}  // namespace im2win
