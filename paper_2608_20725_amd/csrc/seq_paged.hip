// Attention of one new token of each sequence over its pages.
//
// The work is the cache's bytes, read once.  The G = H/Hkv queries of a
// key/value head are columns of the 16x16 matrix instructions, 16 to a wave; a
// wave streams tiles of 32 or 64 keys straight from the pages into its operand
// registers, with no copy in LDS and no barrier between the waves:
//   scores  [key][query]: a lane's 16 bytes of a key are the operand as they lie
//           (the order of channels within a product is free, q follows it);
//   output  [channel][query]: the scores' registers are the operand as they lie,
//           and a lane holds DP/16 channels of KEYS/4 keys, which it turns from
//           rows of keys into rows of channels by byte permutations.
// While a tile's scores are made the values are on their way, and while the
// values are summed the next keys.  The four waves of a workgroup take tiles in
// turn; where a head has more than 16 queries, two or four of them take the
// same tile for 16 queries each, so that memory still gives it once.  All keys
// are shared evenly between the workgroups; the parts of a sequence (maximum,
// sum, output) are joined in LDS and by paged_join.
//
// 8-bit pages go through the matrix cores as fp16, which holds every code
// exactly; a key's scale multiplies its score, a value's the probability, over
// the power of two at or above the largest such product so far (not the largest
// scale: a value that is not looked at would take the others' bits).  bf16 and fp32
// queries over them are brought to fp16's range by a power of two a row: what
// falls below 2^-39 of the row's largest channel is lost, less than fp32 sums
// lose.  fp32 ones, and their probabilities, are two fp16 numbers each, 22 bits,
// at a quarter of the fp32 instructions' time; probabilities over 16-bit pages are
// two numbers of the pages' type.
#include "seq_attn.hpp"
#include "seq_cache.hpp"

namespace im2win {
namespace {

constexpr int kWavesP = 4;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

// 8 bytes between rows are certain, 16 only where D is a multiple of 16.
typedef u32x4_t u32x4_a8 __attribute__((aligned(8)));
typedef f32x8_t f32x8_a16 __attribute__((aligned(16)));

template <bool B, class X, class Y>
struct Pick {
    typedef X T;
};
template <class X, class Y>
struct Pick<false, X, Y> {
    typedef Y T;
};

struct F32Wide {  // fp32 operands, v_mfma_f32_16x16x4_f32
    typedef float elem;
};

// ---- codes to fp16, exact ----
// Two codes, bytes A and B (0 .. 3 of x, 4 .. 7 of y), as two halves of a word.
template <class Code>
struct Half;
template <>
struct Half<CodeI8> {
    // 1024 + (code + 128) by its bits, minus 1152
    template <int A, int B>
    __device__ static inline uint32_t two(uint32_t y, uint32_t x)
    {
        const uint32_t w = __builtin_amdgcn_perm(y, x, 0x0C000C00u | (B << 16) | A);
        const h2 less = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        return __builtin_bit_cast(uint32_t, (h2)(__builtin_bit_cast(h2, w ^ 0x64806480u) + less));
    }
};
template <>
struct Half<CodeE4M3> {
    template <int A, int B>
    __device__ static inline uint32_t two(uint32_t y, uint32_t x)
    {
        if constexpr (A % 4 == 0 && B == A + 1)
            return of<false>(A ? y : x);
        else if constexpr (A % 4 == 2 && B == A + 1)
            return of<true>(A > 3 ? y : x);
        else
            return of<false>(__builtin_amdgcn_perm(y, x, 0x0C0C0000u | (B << 8) | A));
    }
    template <bool UPPER>
    __device__ static inline uint32_t of(uint32_t w)
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, UPPER));
    }
};

// Keys of a tile, of `bytes` each in a page: two sizes, but for 16 bits and 128
// channels, whose products take 32 keys at once.
constexpr int tile_keys(int64_t bytes, bool small) { return bytes <= 128 ? (small ? 32 : 64) : bytes > 256 && small ? 16 : 32; }

// ---- the two products ----
// E: type of the queries; Code: CodeI8, CodeE4M3 or void (pages of E itself); DP:
// channels, 64 or 128, of which a head has D; SMALL: the smaller tiles.
template <class E, class Code, int DP, bool SMALL>
struct Math {
    static constexpr bool kCodes = !__is_same(Code, void);
    static constexpr bool kWide = __is_same(E, EltF32) && !kCodes;  // fp32 instructions
    static constexpr bool kHalf = kCodes || __is_same(E, EltF16);   // fp16 operands
    static constexpr bool kRange = kCodes && !__is_same(E, EltF16); // queries brought to fp16's range
    static constexpr int kTerms = kCodes && __is_same(E, EltF32) ? 2 : 1;  // operands a query's number
    // Operands a weight.  In one, 16 bits wide, a weight is off by as much as a 16-bit
    // result; a second, for what the first leaves, takes no time that is seen, as the
    // matrix cores wait for memory: 32 caches of up to 8192, 8 heads, one and two: bf16 of
    // 128 channels 131 and 131 us, of 64 65 and 65, of 96 103 and 104; 64 heads over one 44
    // and 45.  Over 8-bit pages, where a value's code is off by 2^-8 of its head's largest,
    // 16-bit queries stay with one, 2^-11: 64 channels 44 and 46 us, 48 caches of up to
    // 16384 214 and 217.
    static constexpr int kWeightTerms = kWide ? 1 : kCodes ? kTerms : 2;
    typedef typename Pick<kWide, F32Wide, typename Pick<kHalf, F16Op, BF16Op>::T>::T Op;
    static constexpr int ES = kCodes ? 1 : kWide ? 4 : 2;
    static constexpr int NK = DP * ES / 64;  // pieces of 16 bytes of a key that a lane takes: bytes 64*c + 16*group
    static constexpr int EPC = 16 / ES;      // channels of a piece
    static constexpr int VC = DP / 16;       // channels of a value that a lane takes: VC*(lane % 16) on
    // A tile's bytes are what a wave keeps on its way: 64 keys where they are short.
    // 48 caches of up to 16384 tokens, 64 heads of 128 over 8, int8 under bf16: 362
    // us with tiles of 32 keys, 245 with 64.  Where a tile a wave is all there is to
    // do, 32 are done sooner: one cache of 2000, 16 heads of 64 over 4, fp16: 7.9 us
    // with 64, 6.6 with 32.
    static constexpr int KEYS = tile_keys(DP * ES, SMALL);
    static constexpr int N = KEYS / 4;       // keys of a lane: 16*(i >> 2) + 4*group + (i & 3)

    struct __attribute__((aligned(VC * ES < 16 ? VC * ES : 16))) Value {
        uint32_t w[VC * ES / 4];
    };
    // A lane's channels of a query: piece by piece, EPC each.
    struct Query {
        typename Op::elem x[kTerms][NK * EPC];
    };
    struct Weights {
        float p[N];
        u32x4_t packed[kWeightTerms][N > 8 ? N / 8 : 1];
    };

    __device__ static inline void set(Query &q, int at, float x)
    {
        q.x[0][at] = (typename Op::elem)x;
        if constexpr (kTerms == 2)
            q.x[1][at] = (typename Op::elem)(x - (float)q.x[0][at]);
    }
    __device__ static inline auto eight(const Query &q, int t, int at)
    {
        typename Op::v8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = q.x[t][at + e];
        return v;
    }
    // Of the pieces FROM .. TO - 1.
    template <int FROM = 0, int TO = NK>
    __device__ static inline f32x4_acc dot(const u32x4_t (&k)[NK], const Query &q, int bytes)
    {
        f32x4_acc s = {0, 0, 0, 0};
#pragma unroll
        for (int c = FROM; c < TO; ++c) {
            if (64 * c >= bytes)  // behind a head's last channel
                break;
            if constexpr (kWide) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)k[c][e]), q.x[0][4 * c + e],
                                                             s, 0, 0, 0);
            } else if constexpr (!kCodes) {
                s = Op::mfma16(__builtin_bit_cast(typename Op::v8, k[c]), eight(q, 0, 8 * c), s);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t x = k[c][2 * h], y = k[c][2 * h + 1];
                    typedef Half<Code> T;
                    const u32x4_t w = {T::template two<0, 1>(y, x), T::template two<2, 3>(y, x),
                                       T::template two<4, 5>(y, x), T::template two<6, 7>(y, x)};
#pragma unroll
                    for (int t = 0; t < kTerms; ++t)
                        s = Op::mfma16(__builtin_bit_cast(typename Op::v8, w), eight(q, t, 16 * c + 8 * h), s);
                }
            }
        }
        return s;
    }

    __device__ static inline void pack(Weights &w)
    {
        if constexpr (!kWide) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                float a = w.p[2 * i], b = w.p[2 * i + 1];
#pragma unroll
                for (int t = 0; t < kWeightTerms; ++t) {
                    const uint32_t x = Op::bits(a), y = Op::bits(b);
                    w.packed[t][i / 4][i % 4] = x | y << 16;
                    if constexpr (kWeightTerms == 2) {
                        a -= (float)__builtin_bit_cast(typename Op::elem, (uint16_t)x);
                        b -= (float)__builtin_bit_cast(typename Op::elem, (uint16_t)y);
                    }
                }
            }
        }
    }
    // Channel VC*(lane % 16) + J of eight of the lane's keys: a row of the operand.
    template <int J>
    __device__ static inline u32x4_t channel(const Value *v)
    {
        u32x4_t w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (ES == 2)
                w[i] = __builtin_amdgcn_perm(v[2 * i + 1].w[J / 2], v[2 * i].w[J / 2], J % 2 ? 0x07060302u : 0x05040100u);
            else
                w[i] = Half<Code>::template two<J % 4, 4 + J % 4>(v[2 * i + 1].w[J / 4], v[2 * i].w[J / 4]);
        }
        return w;
    }
    // o[j] += channel j of the values times their weights.
    template <int J = 0>
    __device__ static inline void sum(f32x4_acc (&o)[VC], const Value (&v)[N], const Weights &w)
    {
        if constexpr (kWide) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                o[J] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, v[i].w[J]), w.p[i], o[J], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < N / 8; ++i) {
                const auto x = __builtin_bit_cast(typename Op::v8, channel<J>(v + 8 * i));
#pragma unroll
                for (int t = 0; t < kWeightTerms; ++t)
                    o[J] = Op::mfma16(x, __builtin_bit_cast(typename Op::v8, w.packed[t][i]), o[J]);
            }
        }
        if constexpr (J + 1 < VC)
            sum<J + 1>(o, v, w);
    }
};

// What the lanes of a wave tell each other of a tile: where its keys and values
// lie (bytes from the head's first), and 8-bit pages' scales.
template <int KEYS, int HEADS>
struct Where {
    int64_t k[KEYS], v[KEYS];
    float ks[HEADS][KEYS], vs[HEADS][KEYS];
};

// ---- how the keys are split ----
// All workgroups take about the same number of keys, whichever sequence they
// belong to: with a share of total/most_parts keys (whole steps) or, where that
// is little, twice as many, a sequence of n keys makes ceil(n/share) parts of
// equal size.  The lengths are known on the GPU only, so each wave adds them up
// and finds its part by a scan over the sequences' counts.
struct Cut {
    int32_t parts, piece;  // parts of a sequence, keys of each (the last has what is left)
};
// x up to a multiple of a step, a power of two.
__device__ inline uint32_t up_to(uint32_t x, int32_t unit) { return (x + unit - 1) & ~(uint32_t)(unit - 1); }
__device__ inline Cut cut_of(int32_t n, int32_t share, int32_t unit)
{
    Cut c = {0, unit};
    if (n > 0) {
        const uint32_t p = (uint32_t)(n - 1) / (uint32_t)share + 1;
        c.piece = (int32_t)up_to((n + p - 1) / p, unit);
        c.parts = (int32_t)((uint32_t)(n - 1) / (uint32_t)c.piece + 1);
    }
    return c;
}

__device__ inline int32_t tokens_of(const Pool &c, const PagedArgs &a, int b)
{
    return b < a.B && c.pages > 0 ? held_tokens(a.len[b], c.max_pages, c.page.d) : 0;
}

__device__ inline int32_t share_of(const Pool &c, const PagedArgs &a, int32_t unit, int lane)
{
    int64_t total = 0;
    for (int b = lane; b < a.B; b += 64)
        total += tokens_of(c, a, b);
    for (int m = 1; m < min(a.B, 64); m <<= 1)  // lanes from B on hold zeros
        total += __shfl_xor((long long)total, m);
    total = (int64_t)__builtin_amdgcn_readfirstlane((int)(total >> 32)) << 32 |
            (uint32_t)__builtin_amdgcn_readfirstlane((int)total);
    // one round of workgroups where that leaves each a few tiles only, two else
    auto of = [&](const FastDiv &parts) {  // ceil(total / parts), at least 1
        if (total <= (int64_t)parts.d)
            return (int64_t)1;
        return total <= (int64_t)UINT32_MAX ? (int64_t)fdiv((uint32_t)(total - 1), parts) + 1 : (total - 1) / parts.d + 1;
    };
    int64_t aim = of(a.half);
    uint32_t most = a.half.d;
    if (aim > 8 * a.row_waves * unit)
        aim = of(a.most), most = a.most.d;
    // no sequence is longer than 2^30
    int32_t share = (int32_t)up_to(aim < 1 << 30 ? (uint32_t)aim : 1u << 30, unit);
    // Sequences end within a share, so that more parts come out, and the few behind
    // the last round take as long as a round of their own: the share grows until its
    // parts (those of half its size or more, others find room between them) are no
    // more than asked for.  Two rounds of short parts even out by themselves.  32
    // caches of up to 8192, 8 heads, without and with this: 64 channels, int8 53 and
    // 44 us, 80, fp16 117 and 106; 16 of 4096, 12 heads of 64, fp32 49 and 45, fp16 30
    // and 28.
    const bool tight = most == a.half.d ? share > 2 * unit : share >= 8 * unit;
    const float limit = 2.0f * (float)share;
    for (int i = 0; tight && i < 3 && share < 1 << 28; ++i) {
        int32_t parts = 0;
        for (int b = lane; b < a.B; b += 64) {
            const int32_t n = tokens_of(c, a, b);
            parts += n > share / 2 ? cut_of(n, share, unit).parts : 0;
        }
        for (int m = 1; m < min(a.B, 64); m <<= 1)
            parts += __shfl_xor(parts, m);
        parts = __builtin_amdgcn_readfirstlane(parts);
        if ((uint32_t)parts <= most)
            break;
        share = (int32_t)up_to((uint32_t)fminf((float)share * (float)parts / (float)most, limit), unit);
    }
    return share;
}

// Parts of the 64 sequences from `base` on: the lane's cut, its tokens, the
// parts up to it and of all.
struct Scan {
    Cut cut;
    int32_t n, upto, all;
};
__device__ inline Scan scan_parts(const Pool &c, const PagedArgs &a, int base, int32_t share, int32_t unit, int lane)
{
    Scan s;
    s.n = tokens_of(c, a, base + lane);
    s.cut = cut_of(s.n, share, unit);
    s.upto = s.cut.parts;
    for (int m = 1; m < min(a.B, 64); m <<= 1) {
        const int32_t below = __shfl_up(s.upto, m);
        s.upto += lane >= m ? below : 0;
    }
    s.all = __builtin_amdgcn_readlane(s.upto, min(a.B, 64) - 1);  // of fewer sequences, lanes beyond them were not added to
    return s;
}

// Part `index` of all sequences' parts in order: keys lo .. hi - 1 of sequence
// b of n keys.  b < 0: there is none.
struct Part {
    int32_t b, n, lo, hi, parts;  // parts of the sequence
};
__device__ inline Part find_part(const Pool &c, const PagedArgs &a, int32_t index, int32_t unit, int lane)
{
    Part p = {-1, 0, 0, 0, 0};
    const int32_t share = share_of(c, a, unit, lane);
    for (int base = 0; base < a.B; base += 64) {
        const Scan s = scan_parts(c, a, base, share, unit, lane);
        if (index >= s.all) {
            index -= s.all;
            continue;
        }
        const int l = __builtin_ctzll(__ballot(s.upto > index));
        const int32_t parts = __builtin_amdgcn_readlane(s.cut.parts, l), piece = __builtin_amdgcn_readlane(s.cut.piece, l);
        p.b = base + l;
        p.n = __builtin_amdgcn_readlane(s.n, l);
        p.lo = (index - (__builtin_amdgcn_readlane(s.upto, l) - parts)) * piece;
        p.hi = min(p.n, p.lo + piece);
        p.parts = parts;
        break;
    }
    return p;
}

// The workspace: for each sequence its first part and their number (written by
// the first part's workgroup, for the join), then the parts: sums, maximum, sum of
// the exponentials and, of 8 bits, what 1 in the sums stands for, of row `head` in
// part `index`.
struct FirstPart {
    int32_t index, parts;
};
__host__ __device__ inline int64_t first_part_floats(int64_t B) { return (2 * B + 3) / 4 * 4; }
__device__ inline float *part_of(const PagedArgs &a, int64_t index, int head, int D)
{
    return a.part + first_part_floats(a.B) + (index * a.H + head) * part_floats(D);
}

// Sums of 8-bit values are kept as numbers times a power of two, the unit, up to the
// last step, after the division by the sum of the weights: a result that the type
// holds is reached, however many keys and however large scales led to it.  The least
// unit is that which 2^14 can be divided by; smaller scales' weights are subnormal.
constexpr float kLeastUnit = 0x1p-112f;
// The power of two at or above x, from kLeastUnit to 2^126.
__device__ inline float power_up_to(float x)
{
    const uint32_t bits = (__builtin_bit_cast(uint32_t, fmaxf(x, kLeastUnit)) + 0x7FFFFFu) & 0x7F800000u;
    return __builtin_bit_cast(float, min(bits, 253u << 23));
}
// Of a power of two from 2^-126 to 2^126.
__device__ inline float inverse(float x) { return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, x)); }

// FULL: heads have DP channels, no more tests of where they end.
// PAIR: two key/value heads that lie side by side are taken as one of DP channels
// with the queries of both, at most 16.  A query keeps the products with its own
// head's pieces of the keys, so that nothing passes from head to head.  A tile's
// bytes are doubled for the same scores, whose columns were idle: 32 caches of 2048
// to 8192 tokens, 8 heads, alone and in pairs: fp16 of 64 channels 78 and 67 us, of
// 32 54 and 39; 34 of up to 13781, 4 heads of 32, fp32 111 and 83; 64 of up to
// 16384, 4 heads of 64, int8 under bf16 106 and 90.  fp32 queries of two heads of 64
// have no registers for it, 8-bit heads of 32 no piece each.
template <class E, class Code, int DP, bool FULL, bool SMALL, bool PAIR>
__global__ __launch_bounds__(64 * kWavesP, 2) void paged_attn(Pool c, PagedArgs a)
{
    typedef Math<E, Code, DP, SMALL> M;
    constexpr int KEYS = M::KEYS, N = M::N, VC = M::VC, ES = M::ES;
    // fp16 probabilities are times 2^14, so that those of long rows stay normal numbers
    // (over 8-bit pages the unit of their products with the scales carries it)
    constexpr float kShift = M::kHalf && !M::kCodes ? 14.0f : 0.0f, kUnshift = M::kHalf && !M::kCodes ? 0x1p-14f : 1.0f;
    constexpr int HEADS = PAIR ? 2 : 1;
    static_assert(!PAIR || (FULL && DP * ES >= 128));  // whole pieces a head
    __shared__ __align__(16) Where<KEYS, HEADS> where[kWavesP];
    __shared__ float box[kWavesP][16][DP + 4];
    __shared__ float sm[kWavesP][16], sl[kWavesP][16], su[kWavesP][16];
    const int D = FULL ? DP : c.D, one = D / HEADS;  // channels of the tile, of a head

    // blockIdx: heads fastest, then row tiles, then parts.  Workgroups go to the 8
    // XCDs in turn (id mod 8); all heads of a part run on one (spread 8, else 1)
    // where they share lines, which it then fetches once: keys that do not lie on
    // 128-byte lines, and the scales of several heads beside keys of few bytes.
    // 32 caches of 2048 to 8192 tokens, 8 heads, 16 tokens a page, heads fastest and
    // on one XCD: bf16 of 96 channels 118 and 112 us, int8 of 128 92 and 87; of 256
    // bytes or more bf16 of 128 139 and 140, fp32 of 64 (16 caches of 4096, 12 heads)
    // 45 and 59.
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int turn = blockIdx.x / a.spread, hk = turn % c.Hkv, rest = turn / c.Hkv, rt = rest % a.row_tiles;
    const int index = rest / a.row_tiles * a.spread + blockIdx.x % a.spread;
    if (index >= a.parts)
        return;
    const int step = KEYS * (kWavesP / a.row_waves);  // keys of the workgroup's tiles
    Part part;
    if (a.most_parts) {
        part = find_part(c, a, index, step, lane);
        if (part.b < 0)
            return;
    } else {
        const int n = tokens_of(c, a, index);
        part = Part{index, n, 0, n, 1};
    }
    const int b = part.b, n = part.n, hi = part.hi;
    if (a.most_parts && part.lo == 0 && hk == 0 && rt == 0 && threadIdx.x == 0)
        ((FirstPart *)a.part)[b] = FirstPart{index, part.parts};

    // this lane's query: column r of the wave's
    const int row0 = (rt * a.row_waves) * 16, row = row0 + wave % a.row_waves * 16 + r;
    const float c2 = a.cap * kLog2e;
    const float *const strip = a.strip + (int64_t)min(hk * a.G + row, a.H - 1) * (2 * a.R + 1) + a.R;

    const char *const kp = c.k + hk * c.k_head, *const vp = c.v + hk * c.v_head;
    const int32_t *const table = c.table + b * c.table_stride;
    Where<KEYS, HEADS> &my = where[wave];
    const bool second = PAIR && r >= a.G / 2;  // this lane's query is the second head's

    // A lane is the owner of key lane % KEYS of each tile.
    auto page_at = [&](int k0) {
        const int key = k0 + lane % KEYS;
        return key < hi ? page_of(table, fdiv((uint32_t)key, c.page), c.max_pages, c.pages) : -1;
    };
    auto inside = [&](int k0) {
        const uint32_t key = k0 + lane % KEYS;
        return (int)(key - fdiv(key, c.page) * c.page.d);
    };
    auto scale_at = [&](const char *s, int64_t page, int64_t tok, int id, int in) {
        return id < 0 ? 0.0f : *(const float *)(s + id * page + in * tok);
    };
    // Keys that are not there read page 0 and are left out of what follows.
    auto tell = [&](int id, int in) {
        if (KEYS == 64 || lane < KEYS)
            my.k[lane % KEYS] = id < 0 ? 0 : id * c.k_page + in * c.k_tok;
        if (KEYS == 64 || lane >= 64 - KEYS)
            my.v[lane % KEYS] = id < 0 ? 0 : id * c.v_page + in * c.v_tok;
    };
    u32x4_t kr[KEYS / 16][M::NK];
    typename M::Value vr[N];
    auto load_keys = [&]() {
#pragma unroll
        for (int s = 0; s < KEYS / 16; ++s) {
            const char *const p = kp + my.k[16 * s + r] + 16 * g;
#pragma unroll
            for (int k = 0; k < M::NK; ++k) {
                const int left = D * ES - (64 * k + 16 * g);  // a multiple of 8
                if (!FULL)
                    kr[s][k] = u32x4_t{0, 0, 0, 0};
                if (FULL || left >= 16) {
                    kr[s][k] = *(const u32x4_a8 *)(p + 64 * k);
                } else if (ES == 1 && left > 0) {
                    const u32x2_t w = *(const u32x2_t *)(p + 64 * k);
                    kr[s][k] = u32x4_t{w[0], w[1], 0, 0};
                }
            }
        }
    };
    auto load_values = [&]() {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const char *const p = vp + my.v[16 * (i >> 2) + 4 * g + (i & 3)] + VC * r * ES;
            if (FULL || VC * r < D)
                vr[i] = *(const typename M::Value *)p;
            else
                vr[i] = typename M::Value{};
        }
    };
    auto load_scales = [&](int id, int in, float (&ks)[HEADS], float (&vs)[HEADS]) {
        if constexpr (M::kCodes) {
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                ks[h] = scale_at(c.ks + (HEADS * hk + h) * c.ks_head, c.ks_page, c.ks_tok, id, in);
                vs[h] = scale_at(c.vs + (HEADS * hk + h) * c.vs_head, c.vs_page, c.vs_tok, id, in);
            }
        }
    };

    // The bias of a tile's scores, loaded before its values: loads end in the order
    // they start, so that scores do not wait for the values or for later keys.
    // 32 caches of 2048 to 8192 tokens, 8 heads of 128, bf16: 157 us where scores
    // load it, 137 here.  fp32 queries of 128 channels over 64 keys of 8-bit pages or
    // 32 of their own type have no registers for that: they load it after the
    // products, before the next keys (int8: 125 us, 112 here with spills, 102 so).
    constexpr bool kEarly = !(__is_same(E, EltF32) && DP == 128 && KEYS == (M::kCodes ? 64 : 32));
    float near[N];
    auto load_bias = [&](int k0) {
        if (a.R > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                near[i] = strip[min(max(k0 + 16 * (i >> 2) + 4 * g + (i & 3) - (n - 1), -a.R), 0)];
        }
    };

    f32x4_acc o[VC];
#pragma unroll
    for (int j = 0; j < VC; ++j)
        o[j] = f32x4_acc{0, 0, 0, 0};
    float m = -INFINITY, l = 0;
    float unit = kLeastUnit;  // 8 bits: what 2^14 in the outputs stands for, a power of two

    // The first loads start in the order in which they are needed last: pages'
    // numbers, the query (made into operands while keys and values come), keys.
    const int first = part.lo + wave / a.row_waves * KEYS;
    int id = page_at(first), in = inside(first);
    int id1 = page_at(first + step), in1 = inside(first + step);
    typedef typename E::T V4 __attribute__((ext_vector_type(4)));
    V4 raw[M::NK * M::EPC / 4];
    {
        const typename E::T *const p = (const typename E::T *)(a.q + b * a.q_sb + (hk * a.G + row) * a.q_sh);
#pragma unroll
        for (int k = 0; k < M::NK * M::EPC / 4; ++k) {
            const int ch = (4 * (4 * k / M::EPC) + g) * M::EPC + 4 * k % M::EPC;
            raw[k] = V4{};
            if (row < a.G && ch < D && (!PAIR || second == (ch >= one)))
                raw[k] = *(const V4 *)(p + (PAIR ? ch % one : ch));
        }
    }
    typename M::Query q;
    float c1 = a.cap > 0 ? a.scale / a.cap : a.scale * kLog2e;
    auto make_query = [&]() {
        float x[M::NK * M::EPC];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < M::NK * M::EPC; ++k) {
            x[k] = E::get(raw[k / 4][k % 4]);
            top = max(top, __builtin_bit_cast(uint32_t, x[k]) & 0x7FFFFFFFu);
        }
        float f = 1.0f;
        if constexpr (M::kRange) {
            top = max(top, (uint32_t)__shfl_xor((int)top, 16));
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
            const int e = max((int)(top >> 23) - 127, -100);  // the row's largest becomes 2^14 .. 2^15
            f = __builtin_bit_cast(float, (uint32_t)(127 + 14 - e) << 23);
            c1 *= __builtin_bit_cast(float, (uint32_t)(127 - 14 + e) << 23);
        }
#pragma unroll
        for (int k = 0; k < M::NK * M::EPC; ++k)
            M::set(q, k, x[k] * f);
    };
    // Of 8-bit pages the query is made at once: its conversion takes the registers
    // that the tile's would be waiting in (48 caches of up to 16384 tokens, int8
    // under bf16: 215 us, 221 the other way).
    if (M::kCodes)
        make_query();
    float ks[HEADS] = {}, vs[HEADS] = {};
    if (first < hi) {
        load_scales(id, in, ks, vs);
        tell(id, in);
        wave_lds_handoff();
        load_keys();
        if (kEarly)
            load_bias(first);
        load_values();
    }
    if (!M::kCodes)
        make_query();
    for (int k0 = first; k0 < hi; k0 += step) {
        float s[N];
#pragma unroll
        for (int h = 0; h < KEYS / 16; ++h) {
            if constexpr (PAIR) {
                const f32x4_acc x = M::template dot<0, M::NK / 2>(kr[h], q, D * ES);
                const f32x4_acc y = M::template dot<M::NK / 2>(kr[h], q, D * ES);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[4 * h + i] = second ? y[i] : x[i];
            } else {
                const f32x4_acc x = M::dot(kr[h], q, D * ES);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    s[4 * h + i] = x[i];
            }
        }
        const uint64_t there = __ballot(id >= 0);  // a bit a key
        float kscale[N], vscale[N];
        wave_lds_handoff();
        if constexpr (M::kCodes) {
#pragma unroll
            for (int h = 0; h < HEADS; ++h) {
                my.ks[h][lane % KEYS] = ks[h];
                my.vs[h][lane % KEYS] = vs[h];
            }
            wave_lds_handoff();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                kscale[i] = my.ks[second][16 * (i >> 2) + 4 * g + (i & 3)];
                vscale[i] = my.vs[second][16 * (i >> 2) + 4 * g + (i & 3)];
            }
        }
        if (!kEarly)
            load_bias(k0);
        // the next tile's keys
        id = id1, in = in1;
        tell(id, in);
        wave_lds_handoff();
        const bool more = k0 + step < hi;
        if (more) {
            load_keys();
            load_scales(id, in, ks, vs);
            id1 = page_at(k0 + 2 * step), in1 = inside(k0 + 2 * step);
        }

        // softmax
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // the factors first: a query of 2^120 and a key of 2^-120 may have a score of 1
            float x = s[i] * (M::kCodes ? c1 * kscale[i] : c1);
            if (a.cap > 0) {
                const float far = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * (2.0f * kLog2e)));
                x = c2 * (fabsf(x) < kSmallTanh ? small_tanh(x) : far);
            }
            if (a.R > 0)
                x += near[i] * kLog2e;
            s[i] = x;
        }
        const bool whole = (KEYS == 64 ? ~there : (uint32_t)~there) == 0;
        if (!whole) {
            // keys that are not there: no score, and no value either, whatever was
            // read in their place (their weights are zero)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!((there >> (16 * (i >> 2) + 4 * g + (i & 3))) & 1)) {
                    s[i] = -INFINITY;
                    vr[i] = typename M::Value{};
                }
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < N; ++i)
            top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m, top), base = now == -INFINITY ? 0.0f : now, less = base - kShift;
        float f = __builtin_amdgcn_exp2f(m - base), sum = 0;
        m = now;
        typename M::Weights w;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            w.p[i] = __builtin_amdgcn_exp2f(s[i] - less);
            sum += w.p[i];
            if constexpr (M::kCodes)
                w.p[i] *= vscale[i];
        }
        l = l * f + sum;
        if constexpr (M::kCodes) {
            // the weights' unit: at or above the largest of them, and of those before
            float most = 0;
#pragma unroll
            for (int i = 0; i < N; ++i)
                most = fmaxf(most, fabsf(w.p[i]));
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            f *= unit;
            unit = power_up_to(fmaxf(f, most));
            const float inv = inverse(unit);
            f *= inv;
#pragma unroll
            for (int i = 0; i < N; ++i)
                w.p[i] *= 0x1p14f * inv;
        }
        if (__any(f != 1.0f)) {
#pragma unroll
            for (int j = 0; j < VC; ++j)
                o[j] *= f;
        }
        M::pack(w);
        M::sum(o, vr, w);
        if (more) {
            if (kEarly)
                load_bias(k0 + step);
            load_values();
        }
    }

    // join the waves of each 16 queries
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        sm[wave][r] = m;
        sl[wave][r] = l;
        if constexpr (M::kCodes)
            su[wave][r] = unit;
    }
    __syncthreads();
    // 8 bits: the unit of a row's sum over the waves w0, w0 + row_waves, ..
    auto common = [&](int w0, int r, float top) {
        const float base = top == -INFINITY ? 0.0f : top;
        float u = 0;
        for (int w = w0; w < kWavesP; w += a.row_waves)
            u = fmaxf(u, su[w][r] * __builtin_amdgcn_exp2f(sm[w][r] - base));
        return power_up_to(u);
    };
    float top = -INFINITY;
    for (int w = wave % a.row_waves; w < kWavesP; w += a.row_waves)
        top = fmaxf(top, sm[w][r]);
    float mine = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    if constexpr (M::kCodes)
        mine *= unit * inverse(common(wave % a.row_waves, r, top));
    // this lane's channels are 4*VC*g .. 4*VC*(g + 1) - 1
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < VC; ++j)
            box[wave][r][4 * VC * g + VC * i + j] = o[j][i] * mine;
    __syncthreads();
    // 16 threads a row, 8 channels each
    const int rr = threadIdx.x >> 4, ch = (threadIdx.x & 15) * 8;
    for (int w0 = 0; w0 < a.row_waves; ++w0) {
        const int rw = row0 + 16 * w0 + rr;
        if (rw >= a.G)
            break;
        const int to_ch = PAIR && rw >= a.G / 2 ? ch - one : ch;  // of its head
        float ms = -INFINITY, sum = 0;
        for (int w = w0; w < kWavesP; w += a.row_waves)
            ms = fmaxf(ms, sm[w][rr]);
        const float base = ms == -INFINITY ? 0.0f : ms;
        f32x8_t v = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int w = w0; w < kWavesP; w += a.row_waves) {
            sum += sl[w][rr] * __builtin_amdgcn_exp2f(sm[w][rr] - base);
            if (ch < DP)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] += box[w][rr][ch + e];
        }
        const float value = M::kCodes ? common(w0, rr, ms) * 0x1p-14f : 1.0f;  // of 1 in v
        if (part.parts > 1) {
            float *const to = part_of(a, index, hk * a.G + rw, one);
            if (to_ch >= 0 && to_ch < one)
                *(f32x8_a16 *)(to + to_ch) = v;
            if (to_ch == 0) {
                to[one] = ms;
                to[one + 1] = sum;
                to[one + 2] = value;
            }
        } else {
            const bool none = sum == 0.0f;  // not ms == -inf: all scores may be NaN
            if (to_ch >= 0 && to_ch < one) {
                typedef typename E::T V8 __attribute__((ext_vector_type(8), aligned(16)));
                V8 y;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    y[e] = E::put(none ? 0.0f : v[e] / sum * value);
                *(V8 *)(a.out + b * a.o_sb + (hk * a.G + rw) * a.o_sh + to_ch * sizeof(typename E::T)) = y;
            }
            if (to_ch == 0)
                a.lse[b * a.H + hk * a.G + rw] = none ? -INFINITY : (ms + __log2f(sum * kUnshift)) * kLn2;
        }
    }
}

// Joins the parts of a row: 32 lanes hold its channels, four each, and `groups`
// of them (1 or 8) take its parts in turn.  Rows of one part are done already.
// SHIFTED: weights are times 2^14; UNITS: sums are times a unit (8 bits).
template <class E, bool SHIFTED, bool UNITS>
__global__ __launch_bounds__(256) void paged_join(Pool c, PagedArgs a, int groups)
{
    typedef float v4 __attribute__((ext_vector_type(4)));
    __shared__ v4 sv[8][32];
    __shared__ float sl[8], sm[8], su[8];
    constexpr float kUnshift = SHIFTED ? 0x1p-14f : 1.0f;
    const int rows = a.B * a.H, lane = threadIdx.x & 31, d = lane * 4, group = threadIdx.x >> 5, first = group % groups;
    const int row = blockIdx.x * (8 / groups) + group / groups, live = row < rows;
    const int b = live ? row / a.H : 0, h = live ? row - b * a.H : 0;
    const FirstPart of = ((const FirstPart *)a.part)[b];  // nobody writes it for a sequence without tokens
    const int64_t at = of.index;
    const int parts = live && tokens_of(c, a, b) > 0 ? of.parts : 0;
    if (groups > 1 ? parts == 1 : __all(parts == 1 || !live))  // groups > 1: one row a workgroup
        return;
    // running maximum, sum, outputs and their unit: a part's numbers are loaded at once
    float m = -INFINITY, l = 0, unit = UNITS ? 0x1p-126f : 1.0f;
    v4 v = {0, 0, 0, 0};
    // the unit of two sums, of which the factors f and g become those to it
    auto meet = [&](float &f, float &g, float other) {
        if constexpr (UNITS) {
            f *= unit, g *= other;
            unit = power_up_to(fmaxf(f, g));
            f *= inverse(unit), g *= inverse(unit);
        }
    };
#pragma unroll 4
    for (int k = first; k < parts; k += groups) {
        const float *const p = part_of(a, at + k, h, c.D);
        const float pm = p[c.D], pl = p[c.D + 1], pu = UNITS ? p[c.D + 2] : 1.0f;
        const v4 pv = d < c.D ? *(const v4 *)(p + d) : v4{0, 0, 0, 0};
        const float top = fmaxf(m, pm), base = top == -INFINITY ? 0.0f : top;
        float f = __builtin_amdgcn_exp2f(m - base), g = __builtin_amdgcn_exp2f(pm - base);
        m = top;
        l = l * f + pl * g;
        meet(f, g, pu);
        v = v * f + pv * g;
    }
    if (groups > 1) {
        sv[group][lane] = v;
        if (lane == 0)
            sl[group] = l, sm[group] = m, su[group] = unit;
        __syncthreads();
        if (group)
            return;
        float top = m;
        for (int k = 1; k < 8; ++k)
            top = fmaxf(top, sm[k]);
        const float base = top == -INFINITY ? 0.0f : top;
        float f = __builtin_amdgcn_exp2f(m - base);
        l *= f;
        m = top;
        for (int k = 1; k < 8; ++k) {
            float g = __builtin_amdgcn_exp2f(sm[k] - base);
            l += sl[k] * g;
            meet(f, g, su[k]);
            v = v * f + sv[k][lane] * g;
            f = 1.0f;
        }
    }
    if (!live || parts == 1)
        return;
    const bool none = l == 0.0f;
    if (lane == 0)
        a.lse[row] = none ? -INFINITY : (m + __log2f(l * kUnshift)) * kLn2;
    if (d < c.D) {
        typedef typename E::T V4 __attribute__((ext_vector_type(4)));
        V4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = E::put(none ? 0.0f : v[e] / l * unit);
        *(V4 *)(a.out + b * a.o_sb + h * a.o_sh + d * sizeof(typename E::T)) = y;
    }
}

// Where no sequence can have more than a few steps, a workgroup takes a whole one
// (most_parts 0): a step more takes less than the join's launch.  One sequence of
// 256, 384, 512 and 768 tokens (steps of 128), split and whole, in a graph: 16
// heads of 64 over 4, fp16 10.2, 10.3, 10.3, 10.4 and 6.3, 7.8, 9.2, 11.8 us; 32 of
// 128 over 8, bf16 11.1, 11.2, 11.2, 11.2 and 7.5, 9.3, 10.9, 14.2; four of 8 heads of
// 80, fp32 13.9, 14.1, 14.1, 14.2 and 12.0, 15.8, 19.7, 28.6.  So too from 513
// sequences or 16384 pairs of a sequence and a tile of heads on: each wave's scan over
// the lengths grows with them, and lengths that differ little even out.  One long
// sequence among short ones does not, and is slower whole.  Split and whole, in a
// graph, bf16: 1024 sequences of 1024 tokens, 8 heads over 1 159 and 100 us, 32 over 8
// 885 and 756; of 512 to 2048 202 and 136, 1030 and 958; of 256, one of 16384 90 and
// 253, 435 and 482; 512 sequences of 64 heads of 64 channels 1506 and 1464, 1885 and
// 1846, 713 and 681.  Below, 512 sequences: 70 and 44, 419 and 380; 86 and 68, 506 and
// 490; 59 and 242, 195 and 389.
struct Plan {
    int32_t row_waves, row_tiles, step;
    bool small, pair;
    int64_t most_parts, parts;  // parts: that the lengths can make at most
};
// Workgroups that share the keys, two rounds of the two that fit a CU.  Measured
// with 512, 768, 1024, 1536 and 2048 (bf16, 32 heads over 8, of 128): 32 caches of
// 2048 to 8192 tokens 140, 153, 135, 134, 139 us, 32 of 8192 tokens 199, 227, 202,
// 206, 206, 4 of 2048 to 8192 22, 25, 23, 27, 27, 16 of 1024 to 4096 39, 38, 36, 42,
// 41; 48 of 4096 to 16384, 64 heads over 8, 445, 441, 386, 380, 385; heads of 64, 32 of
// 2048 to 8192, 69, 77, 75, 78, 76.
constexpr int64_t kTarget = 1024;
// pair: heads may be taken by two (see paged_attn).
Plan plan_of(const Pool &c, int ct, int64_t B, int64_t H, int dt, bool pair)
{
    Plan p;
    p.pair = pair;
    const int64_t Hkv = pair ? c.Hkv / 2 : c.Hkv, G = H / Hkv;
    const int64_t bytes = (c.D * (pair ? 2 : 1) <= 64 ? 64 : 128) * (ct != dt ? 1 : dt == IM2WIN_F32 ? 4 : 2);
    p.row_waves = G <= 16 ? 1 : G <= 32 ? 2 : 4;
    p.row_tiles = (int32_t)((G + 16 * p.row_waves - 1) / (16 * p.row_waves));
    const int64_t heads = Hkv * p.row_tiles, most = (int64_t)c.max_pages * c.page.d;
    const int32_t waves = kWavesP / p.row_waves;
    const int32_t least = tile_keys(bytes, true) * waves;
    p.small = B * heads <= kTarget / 2 && (most + least - 1) / least * B * heads <= kTarget / 2;
    p.step = tile_keys(bytes, p.small) * waves;
    // Enough workgroups first: 2000 tokens, 16 heads of 64 over 4, fp16, 9.9 us alone
    // and 10.7 in pairs; 4096, 32 over 8, bf16, 9.8 and 10.5; 2000, 32 over 32, 11.0 and 10.8.
    if (p.small && pair)
        return plan_of(c, ct, B, H, dt, false);
    const int64_t steps = (most + p.step - 1) / p.step;
    const int64_t few = ct == IM2WIN_F32 ? 2 : 4;
    p.most_parts = steps <= few || B > 512 || B * heads >= 16 * kTarget ? 0 : (kTarget + heads - 1) / heads;
    p.parts = p.most_parts ? (p.most_parts + B < B * steps ? p.most_parts + B : B * steps) : B;
    return p;
}
// Whether pairs of heads can be taken as one, wherever they lie.
bool pairs(const Pool &c, int ct, int64_t H, int dt)
{
    return (c.D == 64 ? dt != IM2WIN_F32 : c.D == 32 && ct == dt) && c.Hkv % 2 == 0 && H / c.Hkv <= 8;
}

// Sets a.spread (see paged_attn) and gives the grid.  Parts are rounded up to the 8
// XCDs where that leaves less than 2^32 lanes; B*H < 2^24 alone does.
uint32_t spread_grid(const Pool &c, PagedArgs &a)
{
    const int64_t heads = (int64_t)c.Hkv * a.row_tiles, even = (a.parts + 7) / 8 * 8 * heads;
    const bool share = c.Hkv > 1 && ((c.k_head | c.v_head) % 128 != 0 || c.k_head < 256 || c.v_head < 256);
    a.spread = share && even < (int64_t)1 << 24 ? 8 : 1;
    return (uint32_t)(a.spread == 8 ? even : a.parts * heads);
}

template <class E, class Code, int DP, bool SMALL>
void run_full(uint32_t grid, const Pool &c, const PagedArgs &a, hipStream_t st)
{
    if (c.D == DP)
        paged_attn<E, Code, DP, true, SMALL, false><<<grid, 64 * kWavesP, 0, st>>>(c, a);
    else
        paged_attn<E, Code, DP, false, SMALL, false><<<grid, 64 * kWavesP, 0, st>>>(c, a);
}
template <class E, class Code, int DP>
void run_pair(Pool c, PagedArgs a, hipStream_t st)
{
    c.Hkv /= 2, c.D *= 2, a.G *= 2;
    c.k_head *= 2, c.v_head *= 2;
    const uint32_t grid = spread_grid(c, a);
    paged_attn<E, Code, DP, true, false, true><<<grid, 64 * kWavesP, 0, st>>>(c, a);
}

template <class E, class Code, int DP>
void run_small(bool small, uint32_t grid, const Pool &c, const PagedArgs &a, hipStream_t st)
{
    if constexpr (Math<E, Code, DP, false>::KEYS != Math<E, Code, DP, true>::KEYS)
        if (small)
            return run_full<E, Code, DP, true>(grid, c, a, st);
    run_full<E, Code, DP, false>(grid, c, a, st);
}

template <class E, class Code>
void run(const Plan &p, const Pool &c, PagedArgs a, hipStream_t st)
{
    if constexpr (!__is_same(E, EltF32))
        if (p.pair && c.D == 64)
            run_pair<E, Code, 128>(c, a, st);
    if constexpr (__is_same(Code, void))
        if (p.pair && c.D == 32)
            run_pair<E, Code, 64>(c, a, st);
    if (!p.pair) {
        const uint32_t grid = spread_grid(c, a);
        c.D <= 64 ? run_small<E, Code, 64>(p.small, grid, c, a, st) : run_small<E, Code, 128>(p.small, grid, c, a, st);
    }
    if (a.most_parts) {
        const int64_t rows = (int64_t)a.B * a.H;
        // one row a workgroup and eight: 256 rows of 128 channels 22.8 and 23.6 us, 512 of
        // 64 23.7 and 24.7, 2048 of 128 140 and 140, 8192 512 and 510
        const int groups = rows <= 2048 ? 8 : 1;
        typedef Math<E, Code, 64, false> M;
        paged_join<E, M::kHalf && !M::kCodes, M::kCodes><<<(uint32_t)((rows * groups + 7) / 8), 256, 0, st>>>(c, a, groups);
    }
}

template <class E>
void run_code(const Plan &p, const Pool &c, int ct, const PagedArgs &a, hipStream_t st)
{
    ct == SEQ_I8     ? run<E, CodeI8>(p, c, a, st)
    : ct == SEQ_E4M3 ? run<E, CodeE4M3>(p, c, a, st)
                     : run<E, void>(p, c, a, st);
}

}  // namespace

int64_t paged_part_floats(const Pool &c, int ct, int64_t B, int64_t H, int dt)
{
    // for either order in which heads may lie
    int64_t parts = 0;
    for (int pair = 0; pair <= (int)pairs(c, ct, H, dt); ++pair) {
        const Plan p = plan_of(c, ct, B, H, dt, pair);
        if (p.most_parts && p.parts > parts)
            parts = p.parts;
    }
    return parts ? first_part_floats(B) + parts * H * part_floats(c.D) : 0;
}

hipError_t launch_paged(const Pool &c, int ct, PagedArgs a, int dt, hipStream_t st)
{
    const int64_t bytes = c.D * (ct != dt ? 1 : dt == IM2WIN_F32 ? 4 : 2);  // of a head
    const Plan p = plan_of(c, ct, a.B, a.H, dt, pairs(c, ct, a.H, dt) && c.k_head == bytes && c.v_head == bytes);
    a.most_parts = (int32_t)p.most_parts, a.parts = (int32_t)p.parts;
    a.most = make_fastdiv(p.most_parts ? (uint32_t)p.most_parts : 1);
    a.half = make_fastdiv((a.most.d + 1) / 2);
    a.row_waves = p.row_waves, a.row_tiles = p.row_tiles;
    if (dt == IM2WIN_F32)
        run_code<EltF32>(p, c, ct, a, st);
    else if (dt == IM2WIN_F16)
        run_code<EltF16>(p, c, ct, a, st);
    else
        run_code<EltBF16>(p, c, ct, a, st);
    return hipGetLastError();
}

}  // namespace im2win
