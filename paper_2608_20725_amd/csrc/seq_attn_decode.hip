// Attention forward with few query rows: single tokens over a long cache.
//
// The work is the cache's bytes, read once.  All query rows that share a
// key/value head (Lq queries of H/Hkv heads) are packed into the 32 columns
// of one score tile, and the keys are split: over workgroups (chunks of
// a.chunk keys) and, within one, over the waves, each of which streams tiles
// of 32 keys through a ring of its own in LDS, two tiles deep, with no
// barrier between the waves.  The parts (running maximum, sum and output) are
// joined within the workgroup through LDS and across chunks by attn_join.
// Bound by the cache's bytes: one token each over 32 caches of up to 8192 keys,
// 8 heads of 128, bf16: 148 us, 4.3 TB/s (a large copy moves 4.9).
#include "seq_attn.hpp"

namespace im2win {
namespace {

template <class Op, int DP>
struct Dec {
    typedef Tile<Op, DP> T;
    static constexpr int kKeys = 32;
    static constexpr int kTileBytes = kKeys * T::kRowBytes;
    static constexpr int kNW = kTileBytes > 8192 ? 2 : 4;  // two tiles of K and V a wave: at most 128 KiB
    static constexpr int kSlotBytes = 2 * kTileBytes;
    static constexpr int kLoads = 2 * kTileBytes / 1024;  // of a wave, a tile
};

template <class Op, int DP>
__global__ __launch_bounds__(64 * (Dec<Op, DP>::kNW)) void attn_decode(AttnArgs a)
{
    typedef Dec<Op, DP> F;
    typedef Tile<Op, DP> T;
    constexpr int NW = F::kNW;
    __shared__ __align__(16) char slot0[NW * F::kSlotBytes];
    __shared__ __align__(16) char slot1[NW * F::kSlotBytes];
    __shared__ float sm[NW][32], sl[NW][32];
    __shared__ int kdoc[NW][32];  // documents of a wave's current tile

    // blockIdx: (sequence, head) fastest, then row tiles, then chunks
    const int heads = a.B * a.Hkv;
    const int bh = blockIdx.x % heads, rest = blockIdx.x / heads, rt = rest % a.tiles, chunk = rest / a.tiles;
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv;
    const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = a.Lq * a.G, row = rt * 32 + (lane & 31);
    const bool live = row < rows;
    const int i = row / a.G, hq = hk * a.G + row - i * a.G;  // this lane's query and head
    const int n = keys_of(a, b), pos = i + first_pos(a, n);

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
    const int plo = wave_min(live ? pos : INT32_MAX), phi = wave_max(live ? pos : INT32_MIN);
    const bool seen = live && lim > 0;
    const int dlo = wave_min(seen ? doc : INT32_MAX), dhi = wave_max(seen ? doc : -1);
    const DocRange *const ranges = a.q_doc ? a.k_range + (int64_t)b * ((a.Lk + kDocTile - 1) / kDocTile) : nullptr;
    const float *const strip = a.strip + (live ? hq * a.strip_step : 0);
    float far_l = 0, far_r = 0;
    if (a.R) {
        far_l = strip[0] * kLog2e;
        far_r = strip[2 * a.R] * kLog2e;
    }

    typename Op::v8 q[DP / 16];
    T::held(q, a.q + b * a.q_sb + hq * a.q_sh + (int64_t)i * a.q_st, live, h, a.D);
    const char *const kp = a.k + b * a.k_sb + hk * a.k_sh, *const vp = a.v + b * a.v_sb + hk * a.v_sh;
    const ScoreArgs sc = score_args(a);
    RowState<Op, DP> st;
    st.clear();

    // the wave's tiles of this chunk: first + wave, + NW, ..
    const int end = min(most, (chunk + 1) * a.chunk), first = chunk * a.chunk + wave * F::kKeys;
    char *const my0 = slot0 + wave * F::kSlotBytes, *const my1 = slot1 + wave * F::kSlotBytes;
    auto issue = [&](char *slot, int k0) {
        const int left = k0 < end ? n - k0 : 0;  // past the end: loads of zeros, so that every tile counts alike
        const int64_t at = k0 < end ? k0 : 0;
        T::template dma<F::kKeys, 1>(slot, kp + at * a.k_st, a.k_st, left, a.D, 0, lane);
        T::template dma<F::kKeys, 1>(slot + F::kTileBytes, vp + at * a.v_st, a.v_st, left, a.D, 0, lane);
    };
    auto step = [&](char *slot, char *other, int k0) {
        if (a.q_doc && h == 0)  // no key from n on is read: Lk may end inside the tile
            kdoc[wave][lane] = k0 + lane < n ? a.k_doc[(int64_t)b * a.Lk + k0 + lane] : -1;
        issue(other, k0 + NW * F::kKeys);
        wait_loads<F::kLoads>();
        asm volatile("" ::: "memory");
        bool skip = false;
        TilePairs tp;
        tp.k0 = k0;
        tp.docs_differ = false;
        if (a.q_doc) {
            const DocRange dr = ranges[k0 / kDocTile];
            skip = !(dr.lo <= dhi && dr.hi >= dlo);
            tp.docs_differ = dr.mixed || dlo != dhi || dr.lo != dlo;
        }
        tp.partial = k0 + F::kKeys > least || tp.docs_differ;
        tp.lim = live ? lim : INT32_MAX;
        tp.doc = doc;
        tp.kdoc = kdoc[wave];
        tp.near = tp.inner = false;
        tp.far = 0;
        if (a.R) {
            const bool left = k0 + F::kKeys - 1 - plo <= -a.R, right = k0 - phi >= a.R;
            tp.near = !left && !right;
            tp.far = left ? far_l : right ? far_r : 0.0f;
        }
        const int d0 = k0 + 4 * h - pos;
        if (!skip)
            attend<Op, DP, 1, kAny>(slot, slot + F::kTileBytes, q, st, sc, tp, lane, [&](int x, bool) {
                return strip[min(max(d0 + x, -a.R), a.R) + a.R] * kLog2e;
            });
        // the slot is read before the next loads are started into it
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("" ::: "memory");
    };
    if (first < end)
        issue(my0, first);
    for (int k0 = first; k0 < end; k0 += 2 * NW * F::kKeys) {
        step(my0, my1, k0);
        if (k0 + NW * F::kKeys < end)
            step(my1, my0, k0 + NW * F::kKeys);
    }
    wait_loads<0>();
    asm volatile("" ::: "memory");

    // join the waves: output sums times 2^(m - largest m), channel by channel
    float l = st.l;
    l += __shfl_xor(l, 32);
    if (h == 0) {
        sm[wave][lane] = st.m;
        sl[wave][lane] = l;
    }
    __syncthreads();
    float m = -INFINITY, sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w)
        m = fmaxf(m, sm[w][lane & 31]);
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < NW; ++w)
        sum += sl[w][lane & 31] * __builtin_amdgcn_exp2f(sm[w][lane & 31] - base);
    const float mine = __builtin_amdgcn_exp2f(st.m - base);
    // [channel][wave][column + 1 pad], in slot0 (and slot1 from wave 2 on)
    float *const box = (float *)(wave < NW / 2 ? slot0 : slot1) + (wave % (NW / 2)) * (DP * 33);
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            box[(32 * dt + reg_row(r) + 4 * h) * 33 + (lane & 31)] = st.o[dt][r] * mine;
    __syncthreads();
    const int64_t out_row = ((int64_t)b * a.H + hq) * a.Lq + i;
    const bool none = sum == 0.0f;  // not m == -inf: all scores may be NaN
    if (a.splits > 1) {
        float *const part = a.part + (((int64_t)chunk * heads + bh) * rows + row) * part_floats(a.D);
        if (live && wave == 0 && h == 0) {
            part[a.D] = m;
            part[a.D + 1] = sum;
        }
    } else if (live && wave == 0 && h == 0) {
        a.lse[out_row] = none ? -INFINITY : st.lse(m, sum);
    }
    // a wave takes every NW-th row, a lane its channels
    for (int c = wave; c < 32 && rt * 32 + c < rows; c += NW) {
        const int rr = rt * 32 + c, ii = rr / a.G, hh = hk * a.G + rr - ii * a.G;
        float ms = -INFINITY, s2 = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w)
            ms = fmaxf(ms, sm[w][c]);
#pragma unroll
        for (int w = 0; w < NW; ++w)
            s2 += sl[w][c] * __builtin_amdgcn_exp2f(sm[w][c] - (ms == -INFINITY ? 0.0f : ms));
        for (int d = lane; d < a.D; d += 64) {
            float v = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w)
                v += ((const float *)(w < NW / 2 ? slot0 : slot1))[(w % (NW / 2)) * (DP * 33) + d * 33 + c];
            if (a.splits > 1)
                a.part[(((int64_t)chunk * heads + bh) * rows + rr) * part_floats(a.D) + d] = v;
            else
                ((typename Op::elem *)(a.out + b * a.o_sb + hh * a.o_sh + (int64_t)ii * a.o_st))[d] =
                    (typename Op::elem)(s2 == 0.0f ? 0.0f : v / s2);
        }
    }
}

// Joins the parts of each row: 32 lanes hold its channels, four each, and
// `groups` of 32 lanes (1 or 8) take its parts in turn.  Eight where there are
// few rows of many parts.  Measured, whole calls, one against eight: 16 rows of
// 2000 keys 16.7 -> 10.4 us, 8 rows of 8192 keys 47 -> 23, 128 rows 55 -> 43;
// one stays where rows are many: 8192 rows of the forward pass 41.7 (eight
// 44.3), 18018 fp32 rows 101 (119).
template <class Op>
__global__ __launch_bounds__(256) void attn_join(AttnArgs a, int groups)
{
    typedef float v4 __attribute__((ext_vector_type(4)));
    __shared__ v4 sv[8][32];
    __shared__ float sl[8];
    const int rows = a.Lq * a.G, heads = a.B * a.Hkv, lane = threadIdx.x & 31, d = lane * 4;
    const int group = threadIdx.x >> 5, part = group % groups;
    const int64_t id = (int64_t)blockIdx.x * (8 / groups) + group / groups;  // (sequence, key/value head, row)
    const bool in = id < (int64_t)heads * rows;
    const int bh = in ? (int)(id / rows) : 0, row = in ? (int)(id - (int64_t)bh * rows) : 0;
    const int b = bh / a.Hkv, hk = bh - b * a.Hkv, i = row / a.G, hq = hk * a.G + row - i * a.G;
    const int64_t step = (int64_t)heads * rows * part_floats(a.D);
    const float *const p = a.part + ((int64_t)bh * rows + row) * part_floats(a.D);
    const int parts = a.chunk ? min(a.splits, (keys_of(a, b) + a.chunk - 1) / a.chunk) : a.splits;
    // lanes take the parts' maxima in turn
    float m = -INFINITY;
    for (int c = lane; c < parts; c += 32)
        m = fmaxf(m, p[c * step + a.D]);
#pragma unroll
    for (int x = 16; x >= 1; x >>= 1)
        m = fmaxf(m, __shfl_xor(m, x));
    const float base = m == -INFINITY ? 0.0f : m;
    v4 v = {0, 0, 0, 0};
    float l = 0;
#pragma unroll 4
    for (int c = part; c < parts; c += groups) {
        const float *const q = p + c * step;
        const float f = __builtin_amdgcn_exp2f(q[a.D] - base);
        l += f * q[a.D + 1];
        if (d < a.D)
            v += *(const v4 *)(q + d) * f;
    }
    if (groups > 1) {
        sv[group][lane] = v;
        if (lane == 0)
            sl[group] = l;
        __syncthreads();
        if (group)
            return;
        for (int k = 1; k < 8; ++k) {
            v += sv[k][lane];
            l += sl[k];
        }
    }
    if (!in)
        return;
    const bool none = l == 0.0f;
    const float inv = none ? 0.0f : 1.0f / l;
    if (lane == 0)
        a.lse[((int64_t)b * a.H + hq) * a.Lq + i] =
            none ? -INFINITY : RowState<Op, 32>::lse(m, l);
    if (d < a.D) {
        typedef typename Op::elem V __attribute__((ext_vector_type(4)));
        V o;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            o[e] = (typename Op::elem)(none ? 0.0f : v[e] * inv);
        *(V *)(a.out + b * a.o_sb + hq * a.o_sh + (int64_t)i * a.o_st + d * sizeof(typename Op::elem)) = o;
    }
}

struct Split {
    int32_t tiles, chunk, splits;
};

// Chunks of a multiple of the waves' tiles: at least 4 workgroups for each of
// 256 CUs where the cache is long enough, so that sequences of different
// lengths even out.  Measured with 256, 512, 1024 and 2048 workgroups wanted:
// one cache of 2000 keys, 16 heads of 64 over 4, fp16 10.6, 10.6, 10.4, 10.6 us;
// 32 caches of up to 8192 keys, 32 heads of 128 over 8, bf16 138.5, 143.3,
// 153.4, 168.8; four of them 25, 31, 43, 62: once the chunks fill the chip,
// fewer and longer ones would be ahead.
Split split_of(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t Hkv, int64_t G, int64_t D)
{
    const int64_t unit = dt == IM2WIN_F32 && D > 64 ? 64 : 128;
    Split s;
    s.tiles = (int32_t)((Lq * G + 31) / 32);
    const int64_t groups = B * Hkv * s.tiles;
    int64_t want = (1024 + groups - 1) / (groups > 0 ? groups : 1);
    if (want < 1)
        want = 1;
    int64_t chunk = (Lk + want - 1) / want;
    chunk = (chunk + unit - 1) / unit * unit;
    if (chunk < unit)
        chunk = unit;
    s.chunk = (int32_t)chunk;
    s.splits = (int32_t)((Lk + chunk - 1) / chunk);
    if (s.splits < 1)
        s.splits = 1;
    return s;
}

template <class Op, int DP>
void run(const AttnArgs &a, hipStream_t st)
{
    attn_decode<Op, DP><<<(uint32_t)(a.B * a.Hkv) * a.tiles * a.splits, 64 * Dec<Op, DP>::kNW, 0, st>>>(a);
}

template <class Op>
void run_dim(const AttnArgs &a, hipStream_t st)
{
    a.D <= 32 ? run<Op, 32>(a, st) : a.D <= 64 ? run<Op, 64>(a, st) : a.D <= 96 ? run<Op, 96>(a, st) : run<Op, 128>(a, st);
}

}  // namespace

// Up to two score tiles of rows for a key/value head.  The whole cache is read
// once a score tile here, once a query head by attn_fwd.  Measured, here
// against there: 64 rows (8 queries of 8 heads) over 32 caches of 4096 keys and
// 8 key/value heads 91 us and 204, over one key/value head 28 and 42, 40 fp32
// rows over 2733 keys 16 and 30; beyond, 128 rows (16 queries of 8 heads) over
// 8192 keys 21 and 17, over 8 such caches 53 and 35.  It is the number of heads
// that costs there: single tokens of 128 heads over one key/value head, which
// the rule leaves to attn_fwd, would take 20 us here and take 58 there, over 32
// caches of 4096 keys 65 and 800.
bool attn_few_rows(int64_t Lq, int64_t H, int64_t Hkv) { return Lq <= 32 && Lq * (H / Hkv) <= 64; }

int64_t attn_decode_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D)
{
    const Split s = split_of(dt, B, Lq, Lk, Hkv, H / Hkv, D);
    return s.splits > 1 ? s.splits * B * H * Lq * part_floats(D) * 4 : 0;
}

void launch_attn_join(const AttnArgs &a, int dt, hipStream_t st)
{
    const int64_t rows = (int64_t)a.B * a.H * a.Lq;
    const int groups = rows <= 2048 && a.splits >= 8 ? 8 : 1;
    const uint32_t grid = (uint32_t)((rows * groups + 7) / 8);
    if (dt == IM2WIN_F32)
        attn_join<F32Op><<<grid, 256, 0, st>>>(a, groups);
    else if (dt == IM2WIN_F16)
        attn_join<F16Op><<<grid, 256, 0, st>>>(a, groups);
    else
        attn_join<BF16Op><<<grid, 256, 0, st>>>(a, groups);
}

hipError_t launch_attn_decode(const AttnArgs &a, int dt, hipStream_t st)
{
    AttnArgs b = a;
    const Split s = split_of(dt, a.B, a.Lq, a.Lk, a.Hkv, a.G, a.D);
    b.tiles = s.tiles, b.chunk = s.chunk, b.splits = s.splits;
    dt == IM2WIN_F32 ? run_dim<F32Op>(b, st) : dt == IM2WIN_F16 ? run_dim<F16Op>(b, st) : run_dim<BF16Op>(b, st);
    if (b.splits > 1)
        launch_attn_join(b, dt, st);
    return hipGetLastError();
}

}  // namespace im2win
