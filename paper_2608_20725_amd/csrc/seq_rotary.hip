// Rotary positions: the pair (a, b) of channels at position p becomes
// m*(a cos t - b sin t, a sin t + b cos t), t = p*freq[pair]; the gradient is
// the same with -t.
//
// Angles are counted in turns, as 64-bit fractions: p*freq mod 1 is one integer
// product whose upper bits wrap by themselves, so an angle of position 2^31 is
// as good as one of position 1 (an fp32 product would be off by 2^-24 of
// p*freq, 8e-3 radians at 131072) and needs no reduction beyond its octant.
// Bound by the bytes: each value is read and written once.  A lane takes 16
// bytes of a head's channels and of their partners, and the same channels of up
// to four heads of the token, so that an angle's sine and cosine (30 operations a
// pair) are spread over them; all of it is loaded before the angles are made and
// stored when all of it is turned.  Backward, 8 rows of 4096 tokens, 40 heads of
// 128, bf16: 121 us, 5.5 TB/s (15 more with the angles first, 10 where each head is
// stored before the next is turned).
#include "seq_rotary.hpp"

namespace im2win {
namespace {

constexpr int kThreads = 256;

// Cosine and sine of `turn` * 2^-32 turns.  The residue of the nearest quarter
// is at most pi/4; the first terms left out are below 2e-9 (sine) and 2e-10.
__device__ inline void cos_sin(uint32_t turn, float &c, float &s)
{
    const uint32_t q = (turn + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(turn - (q << 30)) * 1.46291807926715968e-9f;  // 2 pi 2^-32
    const float z = x * x;
    float a = fmaf(z, 1.0f / 362880, -1.0f / 5040), b = fmaf(z, -1.0f / 3628800, 1.0f / 40320);
    a = fmaf(z, a, 1.0f / 120), b = fmaf(z, b, -1.0f / 720);
    a = fmaf(z, a, -1.0f / 6), b = fmaf(z, b, 1.0f / 24);
    a = fmaf(x * z, a, x), b = fmaf(z, b, -0.5f);
    b = fmaf(z, b, 1.0f);
    c = q & 1 ? a : b;
    s = q & 1 ? b : a;
    c = (q + 1) & 2 ? -c : c;
    s = q & 2 ? -s : s;
}

// N values from p on as they lie in memory, vectors with their element's alignment,
// as rotated parts and strides may start anywhere.  PART: fewer, n, may be there.
template <class T, int N, bool PART>
struct Run {
    typedef T V __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    __device__ static inline V load(const char *p, int n)
    {
        if (!PART || n >= N)
            return *(const V *)p;
        V v = {};
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < n)
                v[e] = ((const T *)p)[e];
        return v;
    }
    // Values from..n-1.
    __device__ static inline void store(char *p, int from, int n, const V &v)
    {
        if (from == 0 && (!PART || n >= N)) {
            *(V *)p = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e >= from && (!PART || e < n))
                ((T *)p)[e] = v[e];
    }
};

// Copies n of fewer than W values: vectors of W/2, W/4, .. 1, as n's bits say.
template <class T, int W>
__device__ inline void copy_few(char *o, const char *p, int n)
{
    if constexpr (W > 1) {
        constexpr int H = W / 2;
        if (n & H) {
            typedef T V __attribute__((ext_vector_type(H), aligned(sizeof(T))));
            *(V *)o = *(const V *)p;
            o += H * sizeof(T), p += H * sizeof(T);
        }
        copy_few<T, H>(o, p, n);
    }
}

// Pairs of a unit: 16 bytes of a side (of both, side by side).
template <class E, bool PAIRED>
constexpr int kPairs = (PAIRED ? 8 : 16) / sizeof(typename E::T);
// Pairs of a unit in small calls and of few pairs, see plan_rotary.
constexpr int kFew = 2;

// Lanes: units of a head fastest, then groups of heads, then tokens.  A unit is
// N pairs (N values and their N partners; side by side, 2N values in a row),
// behind them, where x is not y (COPIES), 16 bytes of channels that are copied.
// Where N does not divide the pairs, the last unit is moved back to end with them:
// the pairs it shares with the one before come out alike, so that both may store
// them, unless x is y, where it stores its own only (the others may be turned
// already).  So too the last unit of the copied channels.
// Turned and copied channels share lines of 128 bytes, and are loaded and stored by
// one instruction where both are 16 bytes, so that no line is written in two
// pieces: 15 rows of 2404 tokens, 40 heads of 64, bf16, 16 channels turned, 66 us
// so, 116 where a wave's copies go before its pairs, 101 where they are loaded with
// them and stored before.
template <class E, bool PAIRED, int N, int HEADS, bool COPIES, int PAIRS>
__global__ __launch_bounds__(kThreads) void rotary(RotaryArgs a, TurnsOf<PAIRS> f)
{
    typedef typename E::T T;
    constexpr int W = PAIRED ? 2 * N : N;
    const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
    if (id >= a.lanes)
        return;
    const uint32_t rest = fdiv(id, a.units), unit = id - rest * a.units.d;
    const uint32_t token = fdiv(rest, a.groups), group = rest - token * a.groups.d;
    const uint32_t b = fdiv(token, a.len), t = token - b * a.len.d;
    const char *x = a.x + b * a.x_sb + t * a.x_st;
    char *y = a.y + b * a.y_sb + t * a.y_st;
    const int half = a.rot / 2;
    constexpr int CW = 16 / sizeof(T);  // copied channels of a lane
    constexpr bool ONE = W == CW;       // loaded and stored as pairs are
    constexpr bool PART = N == kFew;    // larger units are for as many pairs or more
    typedef Run<T, N, PART> R;
    typedef Run<T, W, PART> RW;
    typedef Run<T, CW, false> RC;
    typename RW::V w[HEADS];  // the pairs (as ONE, also copied channels, whose bits stay), or their first side and in v the second
    typename R::V v[HEADS];
    typename RC::V copied[HEADS];

    // this lane's heads: group, group + groups, ..
    int copies = COPIES && (int)unit >= a.pair_units;
    const int own = unit * N;  // its pairs are own .. own + N - 1, as far as there are
    const int first = half >= N ? min(own, half - N) : own, n = half - first;
    int at = PAIRED ? 2 * first : first, values = PAIRED ? 2 * n : n;
    const int to = half * sizeof(T);
    if (copies) {
        at = a.rot + (unit - a.pair_units) * CW;
        values = a.D - at;
        if (a.D - a.rot < CW) {
#pragma unroll
            for (int k = 0; k < HEADS; ++k) {
                const int h = group + k * a.groups.d;
                if (h >= a.H)
                    break;
                copy_few<T, CW>(y + h * a.y_sh + at * sizeof(T), x + h * a.x_sh + at * sizeof(T), values);
            }
            return;
        }
        at = min(at, a.D - CW);
        values = CW;
    }
    x += at * sizeof(T);
    y += at * sizeof(T);
    // first, so that the angles need not wait for the rest
    int64_t pos = t;
    if (a.pos)
        pos = a.by_token ? (int64_t)a.pos[token] : (int64_t)a.pos[b] + t;
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = group + k * a.groups.d;
        if (h >= a.H)
            break;
        const char *const p = x + h * a.x_sh;
        if (!ONE && copies)
            copied[k] = *(const typename RC::V *)p;
        else
            w[k] = RW::load(p, values);
        if (!PAIRED && !copies)
            v[k] = R::load(p + to, n);
    }
    if constexpr (COPIES)
        asm("" : "+v"(copies));  // or the compiler makes two paths of it, one behind the other
    float c[N], s[N];
    if (!copies) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const uint64_t turn = (uint64_t)pos * f.turn[e < n ? first + e : 0];
            cos_sin((uint32_t)(turn >> 32), c[e], s[e]);
            c[e] *= a.amplitude;
            s[e] *= a.sin_amplitude;
        }
    }
    const int skip = a.in_place && !copies ? own - first : 0;  // pairs that the unit before stores
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = group + k * a.groups.d;
        if (h >= a.H)
            break;
        if (!copies) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float p = E::get(w[k][PAIRED ? 2 * e : e]);
                const float q = E::get(PAIRED ? w[k][PAIRED ? 2 * e + 1 : 0] : v[k][e]);
                // Rounded to fp32, then to T, wherever in a vector the pair stands: the
                // compiler may neither fuse the products its own way nor make a mixed
                // fp16 instruction of the sum and its conversion.
                float fp = fmaf(p, c[e], -(q * s[e])), fq = fmaf(p, s[e], q * c[e]);
                asm("" : "+v"(fp), "+v"(fq));
                w[k][PAIRED ? 2 * e : e] = E::put(fp);
                if constexpr (PAIRED)
                    w[k][2 * e + 1] = E::put(fq);
                else
                    v[k][e] = E::put(fq);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        const int h = group + k * a.groups.d;
        if (h >= a.H)
            break;
        char *const o = y + h * a.y_sh;
        if (!ONE && copies) {
            *(typename RC::V *)o = copied[k];
        } else if (!PART && skip == 0) {
            *(typename RW::V *)o = w[k];
            if (!PAIRED && !copies)
                *(typename R::V *)(o + to) = v[k];
        } else {
            RW::store(o, PAIRED ? 2 * skip : skip, values, w[k]);
            if (!PAIRED && !copies)
                R::store(o + to, skip, n, v[k]);
        }
    }
}

template <class E, bool PAIRED, bool COPIES, int PAIRS>
void run_copies(const RotaryArgs &a, const TurnsOf<PAIRS> &f, hipStream_t st)
{
    const uint32_t grid = (a.lanes + kThreads - 1) / kThreads;
    const bool heads = (uint32_t)a.H > a.groups.d;  // up to 4 a lane
    if (a.few && heads)
        rotary<E, PAIRED, kFew, 4, COPIES><<<grid, kThreads, 0, st>>>(a, f);
    else if (a.few)
        rotary<E, PAIRED, kFew, 1, COPIES><<<grid, kThreads, 0, st>>>(a, f);
    else if (heads)
        rotary<E, PAIRED, kPairs<E, PAIRED>, 4, COPIES><<<grid, kThreads, 0, st>>>(a, f);
    else
        rotary<E, PAIRED, kPairs<E, PAIRED>, 1, COPIES><<<grid, kThreads, 0, st>>>(a, f);
}

template <class E, bool PAIRED, int PAIRS>
void run(const RotaryArgs &a, const TurnsOf<PAIRS> &f, hipStream_t st)
{
    (int)a.units.d > a.pair_units ? run_copies<E, PAIRED, true>(a, f, st) : run_copies<E, PAIRED, false>(a, f, st);
}

template <class E>
void run_pairs(const RotaryArgs &a, const Turns &f, bool paired, hipStream_t st)
{
    if (a.rot / 2 > kUsualPairs)
        return paired ? run<E, true>(a, f, st) : run<E, false>(a, f, st);
    TurnsOf<kUsualPairs> g;
    for (int i = 0; i < kUsualPairs; ++i)
        g.turn[i] = f.turn[i];
    paired ? run<E, true>(a, g, st) : run<E, false>(a, g, st);
}

}  // namespace

bool plan_rotary(RotaryArgs &a, int64_t B, int64_t L, bool paired, bool in_place, int dt)
{
    const int64_t e = dt == IM2WIN_F32 ? 4 : 2;
    // Where two pairs a lane make 2^17 lanes at most (512 a CU), the time is one
    // lane's: 4 tokens of 40 heads of 128, bf16: 3.8 us with eight pairs, 3.0 with two.
    // Two also where there are fewer than a larger unit has.
    const int64_t units_few = (a.rot / 2 + kFew - 1) / kFew, full = (paired ? 8 : 16) / e;
    const bool small = B * L <= 1 << 17 && B * L * a.H <= 1 << 17 && B * L * a.H * units_few <= 1 << 17;
    a.few = small || a.rot / 2 < full;
    const int64_t N = a.few ? kFew : full, W = 16 / e;
    a.pair_units = (int32_t)((a.rot / 2 + N - 1) / N);
    const int64_t units = a.pair_units + (in_place ? 0 : (a.D - a.rot + W - 1) / W);
    if (B * L * units > UINT32_MAX)  // so that the products below fit
        return false;
    // Heads a lane: 4 where that leaves 2^17 lanes or more, else one.  40 heads of 128,
    // bf16, with one and with four: 16 tokens 2.1 and 3.0 us, 512 4.1 and 4.6, 1024 5.9
    // and 5.9, 4096 16.8 and 13.5, 16384 63.9 and 60.6.
    const int64_t one = B * L * units * a.H;
    int64_t groups = a.H;
    if (one >= (int64_t)1 << 19)
        groups = (a.H + 3) / 4;
    const int64_t lanes = B * L * units * groups;
    if (lanes > UINT32_MAX - kThreads)
        return false;
    a.in_place = in_place;
    a.lanes = (uint32_t)lanes;
    a.units = make_fastdiv((uint32_t)units);
    a.groups = make_fastdiv((uint32_t)groups);
    a.len = make_fastdiv((uint32_t)L);
    return true;
}

hipError_t launch_rotary(const RotaryArgs &a, const Turns &f, bool paired, int dt, hipStream_t st)
{
    if (dt == IM2WIN_F32)
        run_pairs<EltF32>(a, f, paired, st);
    else if (dt == IM2WIN_F16)
        run_pairs<EltF16>(a, f, paired, st);
    else
        run_pairs<EltBF16>(a, f, paired, st);
    return hipGetLastError();
}

}  // namespace im2win
