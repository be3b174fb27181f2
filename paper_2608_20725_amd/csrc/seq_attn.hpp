// What the attention kernels share: operand tiles in LDS, matrix fragments,
// masks and the score function.
//
// All kernels compute score tiles with one token of the *held* side (queries
// in the forward and dq kernels, keys in the dk/dv kernel) per lane and the
// tokens of the *streamed* side down the registers.  In the 32x32 layout of
// the matrix cores lane l holds column l & 31 (its held token) and, with
// h = l >> 5, rows 8*(r/4) + 4*h + r%4 in registers r = 0 .. 15 (streamed
// tokens).  So
//   - a softmax row lies in one lane and its partner l ^ 32: statistics are
//     per-lane scalars, and rescaling the output is one multiply a register;
//   - registers 8*ks .. 8*ks+7 are, as they are, the B operand of the second
//     product over streamed tokens 16*ks .. 16*ks+15 (a product does not
//     depend on the order in which both operands number the summed index), so
//     probabilities never leave the registers;
//   - that product's A operand is the streamed tile transposed, which
//     ds_read_tr16_b64 reads from its row-major copy.
// The streamed tiles (64 tokens, or 32 in fp32) are shared by the workgroup's
// four waves through LDS, in 16-byte chunks permuted within a row (swz) so
// that both ways of reading spread over the banks.
#pragma once

#include "mfma16.hpp"
#include "seq.hpp"

namespace im2win {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kWaves = 4;            // waves a workgroup
constexpr int kHeld = 32 * kWaves;   // held tokens a workgroup
constexpr int kDocTile = 64;         // tokens a document-range record covers

// Document ids of a tile of kDocTile tokens: the range of those >= 0 (lo > hi
// when there are none) and whether the tile holds more than one value.
struct DocRange {
    int32_t lo, hi, mixed, pad;
};

struct AttnArgs {
    const char *q, *k, *v, *o, *dout;
    char *out, *dq, *dk, *dv;
    float *lse;
    float *stat;          // backward: [B][H][2][Lq rounded up to 64] lse*log2(e) less p_shift (+inf: no pair), dout.out
    float *norms;         // backward, fp16: the largest |dout_i| and |v_j| of groups of rows
    float *part;          // sums of rows that several workgroups share
    float *strip_part;    // backward: the strip's gradients of every workgroup
    const float *strip;   // its middle 2R+1 entries
    int64_t strip_step;   // floats between its heads
    const int32_t *kv_len, *prefix, *q_doc, *k_doc;
    const DocRange *q_range, *k_range;  // [B][ceil(L / kDocTile)]
    // byte strides
    int64_t q_sb, q_sh, k_sb, k_sh, v_sb, v_sh, o_sb, o_sh, do_sb, do_sh, dq_sb, dq_sh, dk_sb, dk_sh, dv_sb, dv_sh;
    int32_t q_st, k_st, v_st, o_st, do_st, dq_st, dk_st, dv_st;
    int32_t B, Lq, Lk, H, Hkv, G, D;
    int32_t causal, align_end, R;
    int32_t tiles, splits, chunk;  // held tiles of a head; workgroups that share one; decode: keys of each
    float scale, cap;
};

// fp32 operands beside F16Op and BF16Op: eight 32x32x2 products, the e-th of
// which takes element e of both fragments.
struct F32Op {
    typedef float v8 __attribute__((ext_vector_type(8)));
    typedef float elem;
    __device__ static inline f32x16_acc mfma(v8 a, v8 b, f32x16_acc c)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

template <class Op>
struct OpInfo {
    static constexpr int kElt = sizeof(typename Op::elem);
    static constexpr bool kIs32 = kElt == 4;
    // all exponent bits set: infinity or NaN
    static constexpr uint32_t kExp = kIs32 ? 0x7f800000u : 0;
};

template <class Op>
__device__ inline uint32_t exp_mask();
template <>
__device__ inline uint32_t exp_mask<F16Op>() { return 0x7c007c00u; }
template <>
__device__ inline uint32_t exp_mask<BF16Op>() { return 0x7f807f80u; }
template <>
__device__ inline uint32_t exp_mask<F32Op>() { return 0x7f800000u; }

// A fragment with its infinities and NaN replaced by zeros; `bad` collects
// whether there were any.
template <class Op>
__device__ inline typename Op::v8 finite(typename Op::v8 f, uint32_t &bad)
{
    constexpr int N = OpInfo<Op>::kIs32 ? 8 : 4;
    typedef uint32_t U __attribute__((ext_vector_type(N)));
    U u = __builtin_bit_cast(U, f);
    const uint32_t m = exp_mask<Op>();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (OpInfo<Op>::kIs32) {
            const bool b = (u[i] & m) == m;
            bad |= b;
            u[i] = b ? 0u : u[i];
        } else {
            // exponent + its lowest bit: carries into the sign place of the
            // half when all exponent bits are set
            const uint32_t low = m & (~m + 0x00010001u) & 0x7fff7fffu;  // lowest exponent bit of both halves
            const uint32_t full = ((u[i] & m) + low) & 0x80008000u;
            bad |= full;
            u[i] &= ~((full >> 15) * 0xffffu);
        }
    }
    return __builtin_bit_cast(typename Op::v8, u);
}

template <class Op>
__device__ inline typename Op::v8 pack8(const f32x16_acc &a, int first)
{
    typename Op::v8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (typename Op::elem)a[first + e];
    return v;
}

template <class Op>
__device__ inline void pack16(const f32x16_acc &a, typename Op::v8 (&v)[2])
{
    v[0] = pack8<Op>(a, 0);
    v[1] = pack8<Op>(a, 8);
}

// One streamed tile in LDS: ROWS tokens of DP channels.
template <class Op, int DP>
struct Tile {
    static constexpr int kElt = OpInfo<Op>::kElt;
    static constexpr int kRowBytes = DP * kElt;
    static constexpr int kChunks = kRowBytes / 16;

    // Chunk c of a row lies at place c ^ swz(row).  LDS serves 256 bytes (16
    // chunks) a cycle: 16 lanes that read one chunk of 16 consecutive rows
    // (row_frag), and 32 lanes that read 64 bytes of 4 consecutive rows
    // (col_frag), each find 16 different places modulo 256 bytes.  Measured
    // against three bits that spread over 128 bytes: 44 % of the LDS cycles of
    // the dk/dv kernel (D = 128) were conflicts, none now.
    __device__ static inline int swz(int row)
    {
        if constexpr (kElt == 2 && kChunks == 16)
            return ((row & 3) << 2) | ((row >> 2) & 3);
        else if constexpr (kElt == 2 && kChunks == 8)  // two rows in 256 bytes
            return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
        else if constexpr (kElt == 2)  // 4 and 12 chunks: four rows start in different quarters
            return (row >> 2) & 3;
        else if constexpr (kChunks % 16 == 0)  // fp32: rows r and r + 4 of a column read in different halves
            return (row & 3) | (((row >> 2) & 1) << 3) | (((row >> 3) & 1) << 2);
        else
            return (row >> 1) & 7;
    }

    // Offset of lane `lane` for row_frag: its row (lane & 31) and the place of
    // its first chunk.  Chunks that differ only in bits below kXor bytes lie
    // at offsets that differ in the same bits, the others further on.
    static constexpr int kXor = kElt == 2 ? (kChunks % 16 == 0 ? 256 : kChunks == 8 ? 128 : 64) : kChunks % 16 == 0 ? 256 : 128;
    __device__ static inline uint32_t row_offset(int lane)
    {
        const int row = lane & 31, first = (lane >> 5) * (kElt / 2);
        return row * kRowBytes + ((first ^ swz(row)) << 4);
    }
    __device__ static inline const char *place(const char *t, uint32_t off, int bytes)
    {
        return t + ((off ^ (bytes % kXor)) + bytes / kXor * kXor);
    }

    // Elements 16*s + 8*h .. +7 of row 32*sub + (lane & 31): A or B operand of
    // step s; `off` = row_offset.
    __device__ static inline typename Op::v8 row_frag(const char *t, uint32_t off, int sub, int s)
    {
        t += 32 * sub * kRowBytes;
        if constexpr (kElt == 2) {
            return *(const typename Op::v8 *)place(t, off, 32 * s);
        } else {
            typedef float v4 __attribute__((ext_vector_type(4)));
            const v4 a = *(const v4 *)place(t, off, 64 * s), b = *(const v4 *)place(t, off, 64 * s + 16);
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }

    // Offset of a lane for col_frag.  16 bits: 16 lanes read 4 rows x 16
    // channels, 8 bytes each, of which lane a receives channel a of the four
    // rows.  fp32: a lane reads its channel of row 4*h.
    __device__ static inline uint32_t col_offset(int lane)
    {
        const int h = lane >> 5;
        if constexpr (kElt == 2) {
            const int a = lane & 15, row = 4 * h + (a >> 2), c = 2 * ((lane >> 4) & 1) + ((a & 3) >> 1);
            return row * kRowBytes + ((c ^ swz(row)) << 4) + (a & 1) * 8;
        } else {
            const int d = lane & 31;
            return 4 * h * kRowBytes + (((d >> 2) ^ swz(4 * h)) << 4) + (d & 3) * 4;
        }
    }

    // Channel d = 32*dt + (lane & 31) of the streamed tokens row0 + 4*h +
    // {0..3, 8..11}: A operand over the transposed tile (row0 a multiple of
    // 16); `off` = col_offset.
    __device__ static inline typename Op::v8 col_frag(const char *t, uint32_t off, int row0, int dt)
    {
        t += row0 * kRowBytes;
        if constexpr (kElt == 2) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 lds_s4;
            // 8 rows on, bit 1 of the chunk permutation differs
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4 *)place(t, off, 64 * dt));
            const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_s4 *)(place(t, off ^ 32, 64 * dt) + 8 * kRowBytes));
            typedef short s8 __attribute__((ext_vector_type(8)));
            const s8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(typename Op::v8, v);
        } else {
            typename Op::v8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int row = 8 * (e >> 2) + (e & 3);  // + 4*h: its bits of the permutation are in `off`
                v[e] = *(const float *)(place(t, off ^ (swz(row) << 4), 128 * dt) + row * kRowBytes);
            }
            return v;
        }
    }

    // Four consecutive channels of one token as fp32 (the rare path).
    __device__ static inline void four(const char *t, int row, int d, float *f)
    {
        const char *p = t + row * kRowBytes + (((d * kElt >> 4) ^ swz(row)) << 4) + ((d * kElt) & 15);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            f[e] = (float)((const typename Op::elem *)p)[e];
    }

    // Starts the copy of a tile to LDS by wave `wave` of NW: `valid` tokens from
    // p on (the others, and channels from D on, become zeros).  The loads
    // write LDS in lane order, so the chunk permutation is applied to the
    // addresses.
    template <int ROWS, int NW>
    __device__ static inline void dma(char *t, const char *p, int32_t stride, int valid, int D, int wave, int lane)
    {
        typedef __attribute__((address_space(3))) void *lds_ptr;
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(p, kMaxRecords);
#pragma unroll
        for (int i = 0; i < ROWS * kChunks / (64 * NW); ++i) {
            const int id = (wave + NW * i) * 64 + lane;
            const int row = id / kChunks, c = (id % kChunks) ^ swz(row);
            const uint32_t off = row < valid && c * 16 < D * kElt ? (uint32_t)(row * stride + c * 16) : kOOB;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(t + (wave + NW * i) * 1024), 16, off, 0, 0, 0);
        }
    }

    // Fragments of a held token straight from memory.
    __device__ static inline void held(typename Op::v8 (&f)[DP / 16], const char *row, bool valid, int h, int D)
    {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            typename Op::v8 z = {};
            f[s] = z;
            if (valid && 16 * s + 8 * h < D)
                f[s] = *(const typename Op::v8 *)(row + (16 * s + 8 * h) * kElt);
        }
    }
};

// Starts the copy of 64 words to LDS by one wave; those from `valid` on become
// zeros.
__device__ inline void dma_words(void *t, const void *p, int valid, int lane)
{
    typedef __attribute__((address_space(3))) void *lds_ptr;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(p, kMaxRecords), (lds_ptr)t, 4,
                                             lane < valid ? (uint32_t)lane * 4 : kOOB, 0, 0, 0);
}

__device__ inline int wave_min(int v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        v = min(v, __shfl_xor(v, m));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ inline int wave_max(int v)
{
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        v = max(v, __shfl_xor(v, m));
    return __builtin_amdgcn_readfirstlane(v);
}

// Both lanes of a pair (l, l ^ 32) get the larger of their values.
__device__ inline float pair_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Row of register r of a 32x32 result, + 4*h.
__device__ constexpr int reg_row(int r) { return 8 * (r >> 2) + (r & 3); }

// How products q.k become scores in units of ln 2: x*c1, or capped,
// c2*tanh(x*c1).
struct ScoreArgs {
    float c1, c2;
    bool cap;
};
__device__ inline ScoreArgs score_args(const AttnArgs &a)
{
    return ScoreArgs{a.cap > 0 ? a.scale / a.cap : a.scale * kLog2e, a.cap * kLog2e, a.cap > 0};
}

// tanh(u) for |u| < 1/4: its Taylor series to u^9 (the next term is below 9e-9
// of the value).  1 - 2/(1 + e^2u), which serves the rest, is off by 6e-8
// whatever u is: with scores far below the cap, as most are, that would be an
// error of 1e-5 in the exponent (cap 50).
constexpr float kSmallTanh = 0.25f;
__device__ inline float small_tanh(float u)
{
    const float w = u * u;
    float p = fmaf(w, 62.0f / 2835.0f, -17.0f / 315.0f);
    p = fmaf(w, p, 2.0f / 15.0f);
    p = fmaf(w, p, -1.0f / 3.0f);
    return fmaf(u * w, p, u);
}

// s = tanh(s*c1) of N tiles.  Where all arguments of the wave are small the
// exponential and the reciprocal are left out; which of the two forms a value
// takes depends on itself alone.
template <int N>
__device__ inline void tanh_scores(f32x16_acc (&s)[N], float c1)
{
    float m[4] = {0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[t][r] *= c1;
            m[r & 3] = fmaxf(m[r & 3], fabsf(s[t][r]));
        }
    if (!__any(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])) >= kSmallTanh)) {
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[t][r] = small_tanh(s[t][r]);
    } else {
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float u = s[t][r];
                const float big = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u * (2.0f * kLog2e)));
                s[t][r] = fabsf(u) < kSmallTanh ? small_tanh(u) : big;
            }
    }
}

// A query's running softmax: output sums, maximum (of the pair), sum (of this
// lane's keys), both times 2^kShift.
template <class Op, int DP>
struct RowState {
    // fp16 keeps 5 exponent bits: its probabilities are multiplied by 2^14, so
    // that those of long rows stay normal numbers.  The maximum is raised only
    // when a score passes it by kSlack, so they stay below 2^15.
    static constexpr bool kIs16 = __is_same(Op, F16Op);
    static constexpr float kShift = kIs16 ? 14.0f : 0.0f;
    static constexpr float kSlack = kIs16 ? 1.0f : 8.0f;
    f32x16_acc o[DP / 32];
    float m, l;

    // ln of the sum of exponentials, from a row's maximum and (whole) sum: the
    // shift is taken off the sum, not off the large logarithm.
    __device__ static inline float lse(float m, float l) { return (m + __log2f(l * (kIs16 ? 0x1p-14f : 1.0f))) * kLn2; }

    __device__ inline void clear()
    {
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o[t][r] = 0;
        m = -INFINITY;
        l = 0;
    }
    __device__ inline void rescale(float f)
    {
        l *= f;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                o[t][r] *= f;
    }
};

// What the queries of a wave and one tile of keys have to do with each other
// (uniform but for lim, doc and far).
struct TilePairs {
    int k0;            // first key
    bool partial;      // some pairs are left out
    bool docs_differ;  // .. by documents
    bool near;         // the bias differs within the tile
    bool inner;        // .. and no distance of the tile is beyond the strip
    float far;         // the bias where it does not
    int lim, doc;      // this lane's query: keys below lim, its document
    const int *kdoc;   // documents of the tile's keys
};

// Runs use(i, fragments of step i) for N steps of G fragments from LDS.
// AHEAD: each step's fragments are read while the step before it runs on the
// matrix cores, and buf[0] holds step 0 on entry.  Left to itself the compiler reads every fragment right before
// its product and waits for it, which costs a kernel of one wave a SIMD 12 %
// (the dk/dv kernel, D = 128); where two or more waves share a SIMD they fill
// each other's waits, and the registers are worth more (8192 tokens forward,
// D = 128: spills, 2.2 times the time).
template <class Op, bool AHEAD, int N, int G, class Load, class Use>
__device__ inline void pipeline(typename Op::v8 (&buf)[2][G], Load load, Use use)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (AHEAD) {
            if (i + 1 < N)
                load(i + 1, buf[(i + 1) & 1]);
            __builtin_amdgcn_sched_barrier(0);
        } else {
            load(i, buf[i & 1]);
        }
        use(i, buf[i & 1]);
    }
}

// Keeps what follows from x inside the loop it stands in: the fragments'
// addresses cost one xor each, and as loop constants a register each.
__device__ inline uint32_t opaque(uint32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Which scores a kernel instance handles: products alone, capped ones, or
// whatever the arguments say (a bias; fp32).  The first two leave out the
// branches and registers of the rest.
enum Feat { kPlain = 0, kCapped = 1, kAny = 2 };

// One tile of 32*SUB keys: s = K q, the softmax's update, o += V^T p.
// near(x, clamp): bias of key x + 4*h of the tile, its distance clamped to the
// strip if `clamp`.
template <class Op, int DP, int SUB, int FEAT, class Near>
__device__ inline void attend(const char *tk, const char *tv, const typename Op::v8 (&q)[DP / 16], RowState<Op, DP> &st,
                              const ScoreArgs &sc, const TilePairs &tp, int lane, Near near)
{
    typedef Tile<Op, DP> T;
    typedef RowState<Op, DP> S;
    typedef typename Op::v8 V8;
    const int h = lane >> 5;
    const uint32_t roff = opaque(T::row_offset(lane)), coff = opaque(T::col_offset(lane));
    const bool cap = FEAT == kAny ? sc.cap : FEAT == kCapped;
    f32x16_acc s[SUB];
#pragma unroll
    for (int t = 0; t < SUB; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s[t][r] = 0;
#pragma unroll
    for (int x = 0; x < DP / 16; ++x)
#pragma unroll
        for (int t = 0; t < SUB; ++t)
            s[t] = Op::mfma(T::row_frag(tk, roff, t, x), q[x], s[t]);

    // A score is s*mul + add (mul > 0): the maximum is taken of s, and one
    // fused multiply-add scales a score and subtracts the maximum.
    float mul = sc.c1, add = FEAT == kAny ? tp.far : 0.0f;
    if (cap) {
        tanh_scores(s, sc.c1);
        mul = sc.c2;
    }
    if ((FEAT == kAny && tp.near) || !(mul > 0)) {
#pragma unroll
        for (int t = 0; t < SUB; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[t][r] = fmaf(s[t][r], mul, add);
        mul = 1.0f;
        add = 0.0f;
    }
    if (FEAT == kAny && tp.near) {
        if (tp.inner) {
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] += near(32 * t + reg_row(r), false);
        } else {
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] += near(32 * t + reg_row(r), true);
        }
    }
    if (tp.partial) {
        const int last = tp.lim - tp.k0 - 4 * h;
#pragma unroll
        for (int t = 0; t < SUB; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                s[t][r] = 32 * t + reg_row(r) < last ? s[t][r] : -INFINITY;
        if (tp.docs_differ)
#pragma unroll
            for (int t = 0; t < SUB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] = tp.kdoc[32 * t + reg_row(r) + 4 * h] == tp.doc ? s[t][r] : -INFINITY;
    }
    // four maxima and sums at a time: no chain of 32 dependent operations
    float m4[4], l4[4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
        m4[x] = s[0][x];
#pragma unroll
    for (int t = 0; t < SUB; ++t)
#pragma unroll
        for (int r = t ? 0 : 4; r < 16; ++r)
            m4[r & 3] = fmaxf(m4[r & 3], s[t][r]);
    float top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
    top = pair_max(fmaf(top, mul, add));
    if (__any(top > st.m + S::kSlack)) {
        // each row by its own scores alone: what a row gives does not depend
        // on the rows beside it
        const bool up = top > st.m + S::kSlack;
        st.rescale(up ? __builtin_amdgcn_exp2f(st.m - top) : 1.0f);
        st.m = up ? top : st.m;
    }
    const float sub = add - (st.m == -INFINITY ? 0.0f : st.m) + S::kShift;
#pragma unroll
    for (int t = 0; t < SUB; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], mul, sub));
            l4[r & 3] = t == 0 && r < 4 ? s[t][r] : l4[r & 3] + s[t][r];
        }
    st.l += (l4[0] + l4[1]) + (l4[2] + l4[3]);

    // P is rounded to 16 bits here, as operand of the matrix cores (fp32 ones
    // run at a seventh of the rate); its sum above and the products' are fp32
    if (!tp.partial) {
#pragma unroll
        for (int i = 0; i < 2 * SUB; ++i) {
            const V8 p = pack8<Op>(s[i >> 1], 8 * (i & 1));
#pragma unroll
            for (int dt = 0; dt < DP / 32; ++dt)
                st.o[dt] = Op::mfma(T::col_frag(tv, coff, 16 * i, dt), p, st.o[dt]);
        }
        return;
    }
    // a value of a left-out pair times its zero must stay zero
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 2 * SUB; ++i) {
        const V8 p = pack8<Op>(s[i >> 1], 8 * (i & 1));
#pragma unroll
        for (int dt = 0; dt < DP / 32; ++dt)
            st.o[dt] = Op::mfma(finite<Op>(T::col_frag(tv, coff, 16 * i, dt), bad), p, st.o[dt]);
    }
    if (__any(bad)) {
        // values that are not finite reach the queries that see them
        for (int kk = 0; kk < 32 * SUB; ++kk) {
            if (tp.k0 + kk >= tp.lim || (tp.docs_differ && tp.kdoc[kk] != tp.doc))
                continue;
#pragma unroll
            for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    float f[4];
                    T::four(tv, kk, 32 * dt + 8 * g + 4 * h, f);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        st.o[dt][4 * g + e] += fabsf(f[e]) < INFINITY ? 0.0f : f[e];
                }
        }
    }
}

// Writes a held token's result times f: channels down the registers of its
// lane pair.
template <class Op, int DP>
__device__ inline void store_row(char *p, const f32x16_acc (&g)[DP / 32], float f, int h, int D)
{
#pragma unroll
    for (int dt = 0; dt < DP / 32; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int d = 32 * dt + 8 * q + 4 * h;
            if (d < D) {
                typedef typename Op::elem V __attribute__((ext_vector_type(4)));
                V v;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = (typename Op::elem)(g[dt][4 * q + e] * f);
                *(V *)(p + d * sizeof(typename Op::elem)) = v;
            }
        }
}

template <int N>
__device__ inline void wait_loads()
{
    // s_waitcnt vmcnt(N), expcnt and lgkmcnt left alone
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// The streamed tiles that hold a document of the workgroup's tokens: one bit
// a tile in `bits` (LDS), 64 tiles a word, `tiles` in all.  Every wave takes
// part; the caller's next barrier publishes them.
__device__ inline void mark_tiles(uint64_t *bits, const DocRange *ranges, int tiles, int tokens, int lo, int hi,
                                  int wave, int lane)
{
    for (int t0 = wave * 64; t0 < tiles; t0 += 64 * kWaves) {
        bool meet = false;
        if (t0 + lane < tiles) {
            const DocRange r = ranges[(t0 + lane) * tokens / kDocTile];
            meet = r.lo <= hi && r.hi >= lo;
        }
        const uint64_t w = __ballot(meet);
        if (lane == 0)
            bits[t0 >> 6] = w;
    }
}

// The first marked tile from t on.
__device__ inline int next_tile(const uint64_t *bits, int t, int tiles)
{
    while (t < tiles) {
        const uint64_t w = bits[t >> 6] >> (t & 63);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)w), hi = __builtin_amdgcn_readfirstlane((uint32_t)(w >> 32));
        if (lo)
            return t + __builtin_ctz(lo);
        if (hi)
            return t + 32 + __builtin_ctz(hi);
        t = (t | 63) + 1;
    }
    return tiles;
}

// The number of keys of sequence b, and the position of its query 0.
__device__ inline int keys_of(const AttnArgs &a, int b)
{
    return a.kv_len ? min(max(a.kv_len[b], 0), a.Lk) : a.Lk;
}
__device__ inline int first_pos(const AttnArgs &a, int n) { return a.align_end ? n - a.Lq : 0; }

// What a workgroup works on: tile `tile` of key/value head `kv` (of B*Hkv) and
// of its query head `g`.  Workgroups go to the 8 XCDs in turn (id mod 8).
//   uneven = false: runs of consecutive ids (head by head) on one XCD, so that
//     the streamed side of a head stays in that XCD's L2.
//   uneven = true (causal masks, whose tiles differ in work): tile 0 of every
//     head first, then tile 1, .., so that the caller can start the longest
//     ones first; heads that share keys still fall on one XCD where the number
//     of key/value heads is a multiple of 8.
struct Work {
    uint32_t kv, g, tile;
};
__device__ inline Work work_item(uint32_t heads, uint32_t G, uint32_t tiles, bool uneven, uint32_t id)
{
    Work w;
    const uint32_t all = heads * G;
    if (uneven) {
        const uint32_t r = id % all;
        w.tile = id / all;
        if (heads % 8 == 0) {
            w.g = r / 8 % G;
            w.kv = r % 8 + 8 * (r / (8 * G));
        } else {
            w.kv = r / G;
            w.g = r % G;
        }
        return w;
    }
    const uint32_t total = all * tiles, x = id % 8, j = id / 8, per = total / 8, rem = total % 8;
    const uint32_t t = x * per + (x < rem ? x : rem) + j;
    w.tile = t % tiles;
    w.kv = t / tiles / G;
    w.g = t / tiles % G;
    return w;
}

// Bytes of AttnArgs::norms and part a call may use.
int64_t attn_norm_bytes(int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv);
int64_t attn_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D, int64_t R,
                        bool backward);
// Distances that occur lie within the longer side, so only that much of a
// strip's range is worth its LDS and its partial gradients.
inline int64_t attn_range(int64_t R, int64_t Lq, int64_t Lk)
{
    const int64_t most = Lq > Lk ? Lq : Lk;
    return R < most ? R : most > 0 ? most : 1;
}

int64_t attn_forward_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D);

// Parts of a row that several workgroups computed: its D output sums, maximum
// and sum, at part[((split*B*Hkv + kv)*Lq*G + query*G + g)*part_floats].
__host__ __device__ inline int64_t part_floats(int64_t D) { return D + 4; }  // D + 2, in 16-byte pieces
void launch_attn_join(const AttnArgs &a, int dt, hipStream_t st);

// Few query rows: the kernel that splits the keys (seq_attn_decode.hip).
bool attn_few_rows(int64_t Lq, int64_t H, int64_t Hkv);
int64_t attn_decode_part_bytes(int dt, int64_t B, int64_t Lq, int64_t Lk, int64_t H, int64_t Hkv, int64_t D);
hipError_t launch_attn_docs(const int32_t *doc, DocRange *out, int64_t B, int64_t L, hipStream_t st);
hipError_t launch_attn_forward(const AttnArgs &a, int dt, hipStream_t st);
hipError_t launch_attn_decode(const AttnArgs &a, int dt, hipStream_t st);
hipError_t launch_attn_backward(const AttnArgs &a, int dt, float *dstrip, hipStream_t st);

}  // namespace im2win
