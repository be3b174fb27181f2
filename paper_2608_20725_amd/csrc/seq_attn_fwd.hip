// Attention forward: one pass over the keys with the running maximum and sum
// of each query's softmax.
//
// A workgroup holds 128 queries of one head (32 a wave, one a lane pair) and
// streams tiles of keys and values:  S^T = K Q^T,  O^T += V^T P^T.
#include "seq_attn.hpp"

namespace im2win {
namespace {

template <class Op, int DP>
struct Fwd {
    typedef Tile<Op, DP> T;
    static constexpr int kKeys = OpInfo<Op>::kIs32 ? 32 : 64;  // keys a tile
    static constexpr int kSub = kKeys / 32;
    static constexpr int kTileBytes = kKeys * T::kRowBytes;
    // fp16 keeps 5 exponent bits: its probabilities are multiplied by 2^14
    // (at most 2^14 then), so that those of long rows stay normal numbers
    static constexpr float kShift = __is_same(Op, F16Op) ? 14.0f : 0.0f;
};

// Does key tile `r` of documents lo .. hi hold a pair with queries of qlo .. qhi?
__device__ inline bool docs_meet(const DocRange &r, int qlo, int qhi) { return r.lo <= qhi && r.hi >= qlo; }

template <class Op, int DP>
__global__ __launch_bounds__(64 * kWaves) void attn_fwd(AttnArgs a)
{
    typedef Fwd<Op, DP> F;
    typedef Tile<Op, DP> T;
    extern __shared__ __align__(16) char lds[];
    char *const tk = lds, *const tv = lds + F::kTileBytes;
    float *const strip = (float *)(lds + 2 * F::kTileBytes);  // 2R+1, times log2(e)
    __shared__ int kdoc[F::kKeys];

    uint32_t qt;
    const uint32_t bh = work_item((uint32_t)(a.B * a.H) * a.tiles, a.tiles, &qt);
    qt = a.tiles - 1 - qt;  // long rows of causal masks first
    const int b = bh / a.H, hq = bh - b * a.H, hk = hq / a.G;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = threadIdx.x >> 6;
    const int i = qt * kHeld + wave * 32 + (lane & 31);  // this lane's query
    const bool live = i < a.Lq;
    const int n = keys_of(a, b);
    const int pos = i + first_pos(a, n);

    // keys below lim take part (with documents: those of the query's document)
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

    if (a.R)
        for (int t = threadIdx.x; t < 2 * a.R + 1; t += 64 * kWaves)
            strip[t] = a.strip[(int64_t)hq * (2 * a.R + 1) + t] * kLog2e;

    // the workgroup's range of keys and documents
    __shared__ int shared_most[kWaves], shared_lo[kWaves], shared_hi[kWaves];
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

    typename Op::v8 q[DP / 16];
    T::held(q, a.q + b * a.q_sb + hq * a.q_sh + (int64_t)i * a.q_st, live, h, a.D);

    const char *kp = a.k + b * a.k_sb + hk * a.k_sh, *vp = a.v + b * a.v_sb + hk * a.v_sh;
    const float c1 = a.cap > 0 ? a.scale / a.cap : a.scale * kLog2e, c2 = a.cap * kLog2e;

    f32x16_acc o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            o[t][r] = 0;
    float m = -INFINITY, l = 0;

    for (int k0 = 0; k0 < wg_most; k0 += F::kKeys) {
        DocRange dr = {0, 0, 0, 0};
        if (a.q_doc) {
            dr = a.k_range[(int64_t)b * ((a.Lk + kDocTile - 1) / kDocTile) + k0 / kDocTile];
            if (!docs_meet(dr, wg_lo, wg_hi))
                continue;
        }
        __syncthreads();  // the tile before this one has been read
        T::template stage<F::kKeys>(tk, kp + (int64_t)k0 * a.k_st, a.k_st, n - k0, a.D);
        T::template stage<F::kKeys>(tv, vp + (int64_t)k0 * a.v_st, a.v_st, n - k0, a.D);
        if (a.q_doc && threadIdx.x < F::kKeys)
            kdoc[threadIdx.x] = k0 + (int)threadIdx.x < n ? a.k_doc[(int64_t)b * a.Lk + k0 + threadIdx.x] : -1;
        __syncthreads();
        if (k0 >= most || (a.q_doc && !docs_meet(dr, dlo, dhi)))
            continue;
        // all pairs of the tile take part?
        const bool docs_differ = a.q_doc && (dr.mixed || dlo != dhi || dr.lo != dlo);
        const bool partial = k0 + F::kKeys > least || docs_differ;

        f32x16_acc s[F::kSub];
#pragma unroll
        for (int t = 0; t < F::kSub; ++t) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[t][r] = 0;
#pragma unroll
            for (int st = 0; st < DP / 16; ++st)
                s[t] = Op::mfma(T::row_frag(tk, 32 * t + (lane & 31), st, h), q[st], s[t]);
        }
        // scores in units of ln 2
#pragma unroll
        for (int t = 0; t < F::kSub; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[t][r] = a.cap > 0 ? c2 * fast_tanh(s[t][r] * c1) : s[t][r] * c1;
        if (a.R) {
            if (k0 + F::kKeys - 1 - plo <= -a.R || k0 - phi >= a.R) {
                const float far = strip[k0 - phi >= a.R ? 2 * a.R : 0];
#pragma unroll
                for (int t = 0; t < F::kSub; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[t][r] += far;
            } else {
                const int d0 = k0 + 4 * h - pos;
#pragma unroll
                for (int t = 0; t < F::kSub; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[t][r] += strip[min(max(d0 + 32 * t + 8 * (r >> 2) + (r & 3), -a.R), a.R) + a.R];
            }
        }
        if (partial) {
            const int last = lim - k0 - 4 * h;
#pragma unroll
            for (int t = 0; t < F::kSub; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * t + 8 * (r >> 2) + (r & 3) >= last)
                        s[t][r] = -INFINITY;
            if (docs_differ)
#pragma unroll
                for (int t = 0; t < F::kSub; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (kdoc[32 * t + 8 * (r >> 2) + 4 * h + (r & 3)] != doc)
                            s[t][r] = -INFINITY;
        }
        // running maximum of the row (both lanes of the pair)
        float top = m;
#pragma unroll
        for (int t = 0; t < F::kSub; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                top = fmaxf(top, s[t][r]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.0f : top;
        const float alpha = __builtin_amdgcn_exp2f(m - base), shifted = base - F::kShift;
        m = top;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o[t][r] *= alpha;
#pragma unroll
        for (int t = 0; t < F::kSub; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(s[t][r] - shifted);
                l += s[t][r];
            }
        uint32_t bad = 0;
#pragma unroll
        for (int t = 0; t < F::kSub; ++t)
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const typename Op::v8 p = pack8<Op>(s[t], 8 * ks);
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt) {
                    typename Op::v8 v = T::col_frag(tv, 32 * t + 16 * ks, dt, lane);
                    if (partial)  // a value of a left-out pair times its zero must stay zero
                        v = finite<Op>(v, bad);
                    o[dt] = Op::mfma(v, p, o[dt]);
                }
            }
        if (partial && __any(bad)) {
            // values that are not finite reach the queries that see them
            for (int kk = 0; kk < F::kKeys; ++kk) {
                if (k0 + kk >= lim || (a.q_doc && kdoc[kk] != doc))
                    continue;
#pragma unroll
                for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float f[4];
                        T::four(tv, kk, 32 * dt + 8 * g + 4 * h, f);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[dt][4 * g + e] += fabsf(f[e]) < INFINITY ? 0.0f : f[e];
                    }
            }
        }
    }

    l += __shfl_xor(l, 32);
    if (!live)
        return;
    const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
    if (h == 0)
        a.lse[((int64_t)b * a.H + hq) * a.Lq + i] = m == -INFINITY ? -INFINITY : (m - F::kShift + __log2f(l)) * kLn2;
    char *op = a.out + b * a.o_sb + hq * a.o_sh + (int64_t)i * a.o_st;
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * h;
            if (d < a.D) {
                typedef typename Op::elem V __attribute__((ext_vector_type(4)));
                V v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = (typename Op::elem)(o[dt][4 * g + e] * inv);
                *(V *)(op + d * T::kElt) = v;
            }
        }
}

// Document ranges, one wave a tile.
__global__ __launch_bounds__(64) void doc_ranges(const int32_t *__restrict__ doc, DocRange *__restrict__ out, int32_t L,
                                                 int32_t tiles)
{
    const int b = blockIdx.x / tiles, t = blockIdx.x - b * tiles, j = t * kDocTile + threadIdx.x;
    const int id = j < L ? max(doc[(int64_t)b * L + j], -1) : -2;
    const int lo = wave_min(id >= 0 ? id : INT32_MAX), hi = wave_max(id);
    const int least = wave_min(id == -2 ? hi : id);
    if (threadIdx.x == 0)
        out[blockIdx.x] = DocRange{lo, hi, least != hi, 0};
}

template <class Op, int DP>
hipError_t run(const AttnArgs &a, hipStream_t st)
{
    typedef Fwd<Op, DP> F;
    const size_t lds = 2 * F::kTileBytes + (a.R ? (2 * a.R + 1) * 4 : 0);
    hipError_t e = hipFuncSetAttribute((const void *)attn_fwd<Op, DP>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                       2 * F::kTileBytes + (2 * SEQ_BIAS_RANGE + 1) * 4);
    if (e != hipSuccess)
        return e;
    AttnArgs b = a;
    b.tiles = (a.Lq + kHeld - 1) / kHeld;
    attn_fwd<Op, DP><<<(uint32_t)(a.B * a.H) * b.tiles, 64 * kWaves, lds, st>>>(b);
    return hipGetLastError();
}

template <class Op>
hipError_t run_dim(const AttnArgs &a, hipStream_t st)
{
    return a.D <= 32 ? run<Op, 32>(a, st)
         : a.D <= 64 ? run<Op, 64>(a, st)
         : a.D <= 96 ? run<Op, 96>(a, st)
                     : run<Op, 128>(a, st);
}

}  // namespace

hipError_t launch_attn_docs(const int32_t *doc, DocRange *out, int64_t B, int64_t L, hipStream_t st)
{
    const int64_t tiles = (L + kDocTile - 1) / kDocTile;
    if (B * tiles == 0)
        return hipSuccess;
    doc_ranges<<<(uint32_t)(B * tiles), 64, 0, st>>>(doc, out, (int32_t)L, (int32_t)tiles);
    return hipGetLastError();
}

hipError_t launch_attn_forward(const AttnArgs &a, int dt, hipStream_t st)
{
    return dt == IM2WIN_F32 ? run_dim<F32Op>(a, st) : dt == IM2WIN_F16 ? run_dim<F16Op>(a, st) : run_dim<BF16Op>(a, st);
}

}  // namespace im2win
