// Attention forward: one pass over the keys with the running maximum and sum
// of each query's softmax.
//
// A workgroup holds 128 queries of one head (32 a wave, one a lane pair) and
// streams tiles of keys and values:  S^T = K Q^T,  O^T += V^T P^T.
// Bound by the vector operations of the softmax (and of a cap) beside the
// matrix cores: 2x8192 causal tokens in 7 documents, 16 query heads of 128 over
// 4, cap 50, bf16: 228 us, 426 TFLOP/s of the pairs that take part.  That is
// with scores below a quarter of the cap, whose tanh is a polynomial; with
// scores that reach it (queries 16 times as large) 291 us on the GPU, 218
// without.
#include "seq_attn.hpp"

namespace im2win {
namespace {

template <class Op, int DP>
struct Fwd {
    typedef Tile<Op, DP> T;
    static constexpr int kSub = OpInfo<Op>::kIs32 ? 1 : 2;
    static constexpr int kKeys = 32 * kSub;  // keys a tile
    static constexpr int kTileBytes = kKeys * T::kRowBytes;
    static constexpr int kOcc = T::kRowBytes <= 128 ? 3 : T::kRowBytes <= 256 ? 2 : 1;  // waves a SIMD to fit in
};

template <class Op, int DP, int FEAT>
__global__ __launch_bounds__(64 * kWaves, (Fwd<Op, DP>::kOcc)) void attn_fwd(AttnArgs a)
{
    typedef Fwd<Op, DP> F;
    typedef Tile<Op, DP> T;
    // two slots, each an array of its own: the compiler can tell that reading
    // one does not wait for the loads that land in the other
    __shared__ __align__(16) char slot0[2 * F::kTileBytes];
    __shared__ __align__(16) char slot1[2 * F::kTileBytes];
    __shared__ int kdoc0[64], kdoc1[64];  // 64: a wave's words
    __shared__ int shared_most[kWaves], shared_lo[kWaves], shared_hi[kWaves];
    extern __shared__ __align__(16) float strip[];  // 2R+1, times log2(e); documents: a bit for each key tile

    // `splits` workgroups share the keys of a query tile
    const Work work = work_item(a.B * a.Hkv, a.G * a.splits, a.tiles, a.causal, blockIdx.x);
    const int qt = a.tiles - 1 - work.tile;  // long rows of causal masks first
    const int g = work.g % a.G, split = work.g / a.G;
    const int b = work.kv / a.Hkv, hk = work.kv - b * a.Hkv, hq = hk * a.G + g;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = qt * kHeld + wave * 32 + (lane & 31);  // this lane's query
    const bool live = i < a.Lq;
    const int n = keys_of(a, b);
    const int pos = i + first_pos(a, n);

    // keys below lim take part (with documents: those of the query's document)
    int lim = n, doc = -1;
    if (a.causal)
        lim = max(0, min(n, max(pos + 1, a.prefix ? a.prefix[b] : 0)));
    if (a.q_doc) {
        if (live)
            doc = a.q_doc[(int64_t)b * a.Lq + i];
        if (doc < 0)
            lim = 0;
    }
    const int most = wave_max(live ? lim : 0), least = wave_min(live ? lim : INT32_MAX);
    const int plo = wave_min(pos), phi = wave_max(pos);
    const bool seen = live && lim > 0;
    const int dlo = wave_min(seen ? doc : INT32_MAX), dhi = wave_max(seen ? doc : -1);

    if (lane == 0) {
        shared_most[wave] = most;
        shared_lo[wave] = dlo;
        shared_hi[wave] = dhi;
    }
    if (FEAT == kAny && a.R)
        for (int t = threadIdx.x; t < 2 * a.R + 1; t += 64 * kWaves)
            strip[t] = a.strip[hq * a.strip_step + t] * kLog2e;
    __syncthreads();
    int wg_most = 0, wg_lo = INT32_MAX, wg_hi = -1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        wg_most = max(wg_most, shared_most[w]);
        wg_lo = min(wg_lo, shared_lo[w]);
        wg_hi = max(wg_hi, shared_hi[w]);
    }
    wg_most = __builtin_amdgcn_readfirstlane(wg_most);
    const int all_tiles = (wg_most + F::kKeys - 1) / F::kKeys;
    const int tiles = (int)((int64_t)all_tiles * (split + 1) / a.splits);  // the first tile not this workgroup's
    const DocRange *const ranges = a.q_doc ? a.k_range + (int64_t)b * ((a.Lk + kDocTile - 1) / kDocTile) : nullptr;
    uint64_t *const bits = (uint64_t *)(strip + (a.R ? 2 * a.R + 2 : 0));
    if (a.q_doc) {
        mark_tiles(bits, ranges, tiles, F::kKeys, wg_lo, wg_hi, wave, lane);
        __syncthreads();
    }

    typename Op::v8 q[DP / 16];
    T::held(q, a.q + b * a.q_sb + hq * a.q_sh + (int64_t)i * a.q_st, live, h, a.D);
    const char *const kp = a.k + b * a.k_sb + hk * a.k_sh, *const vp = a.v + b * a.v_sb + hk * a.v_sh;
    const ScoreArgs sc = score_args(a);
    RowState<Op, DP> st;
    st.clear();

    auto issue = [&](char *slot, int *doc_ids, int t) {
        const int k0 = t * F::kKeys;
        T::template dma<F::kKeys, kWaves>(slot, kp + (int64_t)k0 * a.k_st, a.k_st, n - k0, a.D, wave, lane);
        T::template dma<F::kKeys, kWaves>(slot + F::kTileBytes, vp + (int64_t)k0 * a.v_st, a.v_st, n - k0, a.D, wave,
                                          lane);
        if (a.q_doc && wave == 0)
            dma_words(doc_ids, a.k_doc + (int64_t)b * a.Lk + k0, n - k0, lane);
    };
    auto after = [&](int t) { return a.q_doc ? next_tile(bits, t, tiles) : t; };
    // tile t in `slot` (its loads under way); starts the loads of the next
    // one into `other` and returns it
    auto step = [&](char *slot, int *doc_ids, char *other, int *other_ids, int t) {
        wait_loads<0>();
        ring_barrier();  // everyone's loads have landed, and `other` has been read
        const int next = after(t + 1), k0 = t * F::kKeys;
        if (next < tiles)
            issue(other, other_ids, next);
        DocRange dr = {0, 0, 0, 0};
        if (a.q_doc)
            dr = ranges[k0 / kDocTile];
        if (k0 >= most || (a.q_doc && !(dr.lo <= dhi && dr.hi >= dlo)))
            return next;
        TilePairs tp;
        tp.k0 = k0;
        tp.docs_differ = a.q_doc && (dr.mixed || dlo != dhi || dr.lo != dlo);
        tp.partial = k0 + F::kKeys > least || tp.docs_differ;
        tp.lim = live ? lim : INT32_MAX;
        tp.doc = doc;
        tp.kdoc = doc_ids;
        tp.near = tp.inner = false;
        tp.far = 0;
        if (FEAT == kAny && a.R) {
            const bool left = k0 + F::kKeys - 1 - plo <= -a.R, right = k0 - phi >= a.R;
            tp.near = !left && !right;
            tp.inner = k0 - phi >= -a.R && k0 + F::kKeys - 1 - plo <= a.R;
            if (!tp.near)
                tp.far = strip[right ? 2 * a.R : 0];
        }
        const int d0 = k0 + 4 * h - pos;
        attend<Op, DP, F::kSub, FEAT>(slot, slot + F::kTileBytes, q, st, sc, tp, lane, [&](int x, bool clamp) {
            return strip[(clamp ? min(max(d0 + x, -a.R), a.R) : d0 + x) + a.R];
        });
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

    float l = st.l;
    l += __shfl_xor(l, 32);
    if (!live)
        return;
    if (a.splits > 1) {  // sums as they are; attn_join joins the splits
        float *const part = a.part + (((int64_t)split * a.B * a.Hkv + work.kv) * a.Lq * a.G + (int64_t)i * a.G + g) * part_floats(a.D);
        store_row<F32Op, DP>((char *)part, st.o, 1.0f, h, a.D);
        if (h == 0) {
            part[a.D] = st.m;
            part[a.D + 1] = l;
        }
        return;
    }
    // no pairs: nothing was added.  The maximum does not tell: it passes over
    // NaN, and stays -inf where all scores are NaN
    const bool none = l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
    if (h == 0)
        a.lse[((int64_t)b * a.H + hq) * a.Lq + i] = none ? -INFINITY : st.lse(st.m, l);
    store_row<Op, DP>(a.out + b * a.o_sb + hq * a.o_sh + (int64_t)i * a.o_st, st.o, inv, h, a.D);
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

// Workgroups that share the keys of one query tile, where there are fewer than
// 512 query tiles (two for each of 256 CUs) and the keys are many enough to
// pay for writing and joining the parts; at least 256 keys each.  Measured,
// one workgroup against split: fp16 64 tiles of 1024 keys 21 -> 19 us, bf16 64
// tiles of 4096 keys 102 -> 42, 256 tiles of 4096 110 -> 98; not split, 128
// tiles of 512 keys 19 (26 split), 256 tiles of 2048 42 (49); fp32 144 tiles of
// 1001 keys 121 -> 70, 168 tiles of 784 71 -> 63.
int32_t forward_splits(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H)
{
    const int64_t groups = B * H * ((Lq + kHeld - 1) / kHeld);
    const int64_t enough = dt == IM2WIN_F32 ? 512 : groups < 256 ? 1024 : 4096;
    if (groups <= 0 || groups >= 512 || Lk < enough)
        return 1;
    const int64_t s = (512 + groups - 1) / groups;
    return (int32_t)(s < Lk / 256 ? s : Lk / 256);
}

template <class Op, int DP, int FEAT>
hipError_t run(const AttnArgs &a, hipStream_t st)
{
    typedef Fwd<Op, DP> F;
    const size_t lds = (a.R ? (2 * a.R + 2) * 4 : 0) + (a.q_doc ? (a.Lk + 64 * F::kKeys - 1) / (64 * F::kKeys) * 8 : 0);
    if (lds) {
        const hipError_t e = hipFuncSetAttribute((const void *)attn_fwd<Op, DP, FEAT>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 16 << 10);
        if (e != hipSuccess)
            return e;
    }
    AttnArgs b = a;
    b.tiles = (a.Lq + kHeld - 1) / kHeld;
    constexpr int dt = __is_same(Op, F32Op) ? IM2WIN_F32 : __is_same(Op, F16Op) ? IM2WIN_F16 : IM2WIN_BF16;
    b.splits = forward_splits(dt, a.B, a.Lq, a.Lk, a.H);
    b.chunk = 0;
    attn_fwd<Op, DP, FEAT><<<(uint32_t)(a.B * a.H) * b.tiles * b.splits, 64 * kWaves, lds, st>>>(b);
    if (b.splits > 1)
        launch_attn_join(b, dt, st);
    return hipGetLastError();
}

template <class Op, int DP>
hipError_t run_feat(const AttnArgs &a, hipStream_t st)
{
    if constexpr (!OpInfo<Op>::kIs32) {
        if (!a.R)
            return a.cap > 0 ? run<Op, DP, kCapped>(a, st) : run<Op, DP, kPlain>(a, st);
    }
    return run<Op, DP, kAny>(a, st);
}

template <class Op>
hipError_t run_dim(const AttnArgs &a, hipStream_t st)
{
    return a.D <= 32 ? run_feat<Op, 32>(a, st)
         : a.D <= 64 ? run_feat<Op, 64>(a, st)
         : a.D <= 96 ? run_feat<Op, 96>(a, st)
                     : run_feat<Op, 128>(a, st);
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

int64_t attn_forward_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D)
{
    if (attn_few_rows(Lq, H, Hkv))
        return attn_decode_part_bytes(dt, B, Lq, Lk, H, Hkv, D);
    const int32_t splits = forward_splits(dt, B, Lq, Lk, H);
    return splits > 1 ? splits * B * H * Lq * part_floats(D) * 4 : 0;
}

hipError_t launch_attn_forward(const AttnArgs &a, int dt, hipStream_t st)
{
    if (attn_few_rows(a.Lq, a.H, a.Hkv))
        return launch_attn_decode(a, dt, st);
    return dt == IM2WIN_F32 ? run_dim<F32Op>(a, st) : dt == IM2WIN_F16 ? run_dim<F16Op>(a, st) : run_dim<BF16Op>(a, st);
}

}  // namespace im2win
