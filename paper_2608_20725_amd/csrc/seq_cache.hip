// The paged key/value cache: new tokens into its pages, whole sequences out of
// them, as they are or through numbers of 8 bits.
//
// Both are one pass: a head's D channels of a token are held by LPR lanes, 8
// each, so that the largest magnitude that an 8-bit scale needs is a few
// exchanges between them and nothing is read twice.  Bound by the bytes.
#include "seq_cache.hpp"

namespace im2win {
namespace {

constexpr int kThreads = 256;

// Eight channels as fp32 and as they lie in memory.
template <class E>
struct Eight {
    typedef typename E::T V __attribute__((ext_vector_type(8), aligned(16)));
    __device__ static inline V bits(const char *p) { return *(const V *)p; }
    __device__ static inline void put(char *p, const V &v) { *(V *)p = v; }
    __device__ static inline f32x8_t values(const V &v)
    {
        f32x8_t x;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = E::get(v[e]);
        return x;
    }
    __device__ static inline V rounded(const f32x8_t &x)
    {
        V v;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = E::put(x[e]);
        return v;
    }
};

// The head's scale, from all its lanes' values (the others hold zeros).
template <class Code, int LPR>
__device__ inline float common_scale(const f32x8_t &x)
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = x[e];  // the builtin takes a vector's element for its first
        top = max(top, __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int m = LPR / 2; m >= 1; m >>= 1)
        top = max(top, (uint32_t)__shfl_xor((int)top, m));
    return top >= 0x7F800000u ? __builtin_nanf("") : Code::scale(top);
}

// A copy's row: key/value head, token, sequence, and this lane's channels.
struct Row {
    uint32_t b, t, head;
    int c;
    bool in;
};
template <int LPR>
__device__ inline Row row_of(const Dense &d, int D, uint32_t group)
{
    Row r;
    const uint32_t token = fdiv(group, d.heads);
    r.head = group - token * d.heads.d;
    r.b = fdiv(token, d.len);
    r.t = token - r.b * d.len.d;
    r.c = (threadIdx.x % LPR) * 8;
    r.in = r.b < (uint32_t)d.B && r.c < D;
    return r;
}

// Code: CodeI8, CodeE4M3, or void where the pages hold E itself.
template <class E, class Code, int LPR>
__global__ __launch_bounds__(kThreads) void cache_write(Pool c, Dense d)
{
    typedef Eight<E> X;
    const Row r = row_of<LPR>(d, c.D, blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR);
    const bool there = r.in && (!d.count || (int32_t)r.t < d.count[r.b]);
    typename X::V k = {}, v = {};
    int32_t id = -1, within = 0;
    if (there) {
        k = X::bits(d.k + r.b * d.k_sb + r.t * d.k_st + r.head * d.k_sh + r.c * sizeof(typename E::T));
        v = X::bits(d.v + r.b * d.v_sb + r.t * d.v_st + r.head * d.v_sh + r.c * sizeof(typename E::T));
        const int64_t pos = (int64_t)(d.start ? d.start[r.b] : 0) + r.t;
        if (pos >= 0 && pos <= INT32_MAX) {
            const uint32_t index = fdiv((uint32_t)pos, c.page);
            within = (uint32_t)pos - index * c.page.d;
            id = page_of(c.table + r.b * c.table_stride, index, c.max_pages, c.pages);
        }
    }
    const bool live = id >= 0;
    if constexpr (__is_same(Code, void)) {
        if (live) {
            X::put(c.k + id * c.k_page + within * c.k_tok + r.head * c.k_head + r.c * sizeof(typename E::T), k);
            X::put(c.v + id * c.v_page + within * c.v_tok + r.head * c.v_head + r.c * sizeof(typename E::T), v);
        }
    } else {
        const f32x8_t kx = X::values(k), vx = X::values(v);
        const float ks = common_scale<Code, LPR>(kx), vs = common_scale<Code, LPR>(vx);
        if (live) {
            *(u32x2_t *)(c.k + id * c.k_page + within * c.k_tok + r.head * c.k_head + r.c) = Code::encode(kx, ks);
            *(u32x2_t *)(c.v + id * c.v_page + within * c.v_tok + r.head * c.v_head + r.c) = Code::encode(vx, vs);
            if (r.c == 0) {
                *(float *)(c.ks + id * c.ks_page + within * c.ks_tok + r.head * c.ks_head) = ks;
                *(float *)(c.vs + id * c.vs_page + within * c.vs_tok + r.head * c.vs_head) = vs;
            }
        }
    }
}

template <class E, class Code, int LPR>
__global__ __launch_bounds__(kThreads) void cache_read(Pool c, Dense d)
{
    typedef Eight<E> X;
    const Row r = row_of<LPR>(d, c.D, blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR);
    if (!r.in)
        return;
    int32_t id = -1, within = 0;
    if ((int32_t)r.t < d.count[r.b]) {
        const uint32_t index = fdiv(r.t, c.page);
        within = r.t - index * c.page.d;
        id = page_of(c.table + r.b * c.table_stride, index, c.max_pages, c.pages);
    }
    typename X::V k = {}, v = {};
    if (id >= 0) {
        const char *const kp = c.k + id * c.k_page + within * c.k_tok + r.head * c.k_head;
        const char *const vp = c.v + id * c.v_page + within * c.v_tok + r.head * c.v_head;
        if constexpr (__is_same(Code, void)) {
            k = X::bits(kp + r.c * sizeof(typename E::T));
            v = X::bits(vp + r.c * sizeof(typename E::T));
        } else {
            const float ks = *(const float *)(c.ks + id * c.ks_page + within * c.ks_tok + r.head * c.ks_head);
            const float vs = *(const float *)(c.vs + id * c.vs_page + within * c.vs_tok + r.head * c.vs_head);
            const u32x2_t kw = *(const u32x2_t *)(kp + r.c), vw = *(const u32x2_t *)(vp + r.c);
            k = X::rounded(Code::decode(kw) * ks);
            v = X::rounded(Code::decode(vw) * vs);
        }
    }
    X::put(d.k + r.b * d.k_sb + r.t * d.k_st + r.head * d.k_sh + r.c * sizeof(typename E::T), k);
    X::put(d.v + r.b * d.v_sb + r.t * d.v_st + r.head * d.v_sh + r.c * sizeof(typename E::T), v);
}

int lanes_of(int64_t D) { return D <= 32 ? 4 : D <= 64 ? 8 : 16; }

template <class E, class Code, int LPR>
void run_lanes(bool write, const Pool &c, const Dense &d, hipStream_t st)
{
    const int64_t rows = (int64_t)d.B * d.L * c.Hkv, each = kThreads / LPR;
    const uint32_t grid = (uint32_t)((rows + each - 1) / each);
    if (write)
        cache_write<E, Code, LPR><<<grid, kThreads, 0, st>>>(c, d);
    else
        cache_read<E, Code, LPR><<<grid, kThreads, 0, st>>>(c, d);
}

template <class E, class Code>
void run(bool write, const Pool &c, const Dense &d, hipStream_t st)
{
    const int lanes = lanes_of(c.D);
    lanes == 4   ? run_lanes<E, Code, 4>(write, c, d, st)
    : lanes == 8 ? run_lanes<E, Code, 8>(write, c, d, st)
                 : run_lanes<E, Code, 16>(write, c, d, st);
}

template <class E>
void run_code(bool write, const Pool &c, int ct, const Dense &d, hipStream_t st)
{
    ct == SEQ_I8     ? run<E, CodeI8>(write, c, d, st)
    : ct == SEQ_E4M3 ? run<E, CodeE4M3>(write, c, d, st)
                     : run<E, void>(write, c, d, st);
}

hipError_t launch(bool write, const Pool &c, int ct, const Dense &d, int dt, hipStream_t st)
{
    if (dt == IM2WIN_F32)
        run_code<EltF32>(write, c, ct, d, st);
    else if (dt == IM2WIN_F16)
        run_code<EltF16>(write, c, ct, d, st);
    else
        run_code<EltBF16>(write, c, ct, d, st);
    return hipGetLastError();
}

}  // namespace

// Workgroups of a copy are counted in rows of 32 bits and make less than 2^32 lanes.
bool cache_grid_fits(int64_t B, int64_t L, int64_t Hkv, int64_t D)
{
    return B * L * Hkv < ((int64_t)1 << 32) / lanes_of(D) - kThreads;
}

hipError_t launch_cache_write(const Pool &c, int ct, const Dense &d, int dt, hipStream_t st)
{
    return launch(true, c, ct, d, dt, st);
}

hipError_t launch_cache_read(const Pool &c, int ct, const Dense &d, int dt, hipStream_t st)
{
    return launch(false, c, ct, d, dt, st);
}

}  // namespace im2win
