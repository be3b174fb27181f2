// Internal definitions of the paged key/value cache: what the host side
// (seq_cache_api.cpp) passes to the launches, and the numbers of 8-bit pages.
#pragma once

#include "seq.hpp"
#include "seq_pages.hpp"

namespace im2win {

// A pool of pages and the table of a batch of sequences; strides in bytes.
struct Pool {
    char *k, *v;
    char *ks, *vs;  // fp32 scales of 8-bit pages, else null
    const int32_t *table;
    int64_t table_stride;  // entries
    int64_t k_page, k_tok, k_head, v_page, v_tok, v_head;
    int64_t ks_page, ks_tok, ks_head, vs_page, vs_tok, vs_head;
    FastDiv page;
    int32_t pages, max_pages, Hkv, D;
};

// The dense side of a copy: [B][L][Hkv][D], strides in bytes.
struct Dense {
    char *k, *v;
    int64_t k_sb, k_st, k_sh, v_sb, v_st, v_sh;
    const int32_t *start, *count;  // write: first position and tokens of each sequence; read: count is its length
    int32_t B, L;
    FastDiv len, heads;
};

hipError_t launch_cache_write(const Pool &c, int ct, const Dense &d, int dt, hipStream_t st);
hipError_t launch_cache_read(const Pool &c, int ct, const Dense &d, int dt, hipStream_t st);
// Whether a copy of B sequences of L tokens fits a grid.
bool cache_grid_fits(int64_t B, int64_t L, int64_t Hkv, int64_t D);

struct PagedArgs {
    const char *q;
    char *out;
    float *lse, *part;
    const int32_t *len;
    const float *strip;  // [H][2R+1], or null
    int64_t q_sb, q_sh, o_sb, o_sh;  // bytes
    int32_t B, H, G, R, row_waves, row_tiles, spread;
    int32_t most_parts, parts;  // see Plan
    FastDiv most, half;         // by most_parts and half as many
    float scale, cap;
};

// Floats that the parts of one call take (0: no keys are split).
int64_t paged_part_floats(const Pool &c, int ct, int64_t B, int64_t H, int dt);
hipError_t launch_paged(const Pool &c, int ct, PagedArgs a, int dt, hipStream_t st);

// ---- numbers of 8 bits --------------------------------------------------------------------------------------------
// A token's head is kept as codes times one fp32 scale, at least 2^-126.  With
// `top` its largest magnitude, int8 has scale top/127 and codes rounded to
// nearest even; e4m3 (4 exponent, 3 fraction bits, largest 448) the smallest
// power of two that keeps top within 448, so that the division is exact and
// only the conversion rounds.  A head with a value that is not finite has scale
// NaN.  `top` and codes travel as bits: comparing them as integers puts
// infinities and NaN above every finite magnitude.

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

struct CodeI8 {
    // The largest scale whose 127-fold is finite: one below the quotient of the
    // largest number.
    static constexpr float kMostScale = 0x1.020406p+121f;
    __device__ static inline float scale(uint32_t top)
    {
        return fminf(fmaxf(__builtin_bit_cast(float, top) / 127.0f, 0x1p-126f), kMostScale);
    }
    // Rounds x/s as if the division were exact: n is the nearest number or one
    // beside it, and x - n*s, which the fma does not round (below s it is a
    // multiple of s's last place, or x itself), tells which.
    __device__ static inline int32_t code(float x, float s, float inv)
    {
        float n = __builtin_rintf(x * inv);
        const float r = fmaf(-n, s, x), h = 0.5f * s;
        const bool odd = (int32_t)n & 1;
        if (r > h || (r == h && odd))
            n += 1.0f;
        else if (r < -h || (r == -h && odd))
            n -= 1.0f;
        return (int32_t)fminf(fmaxf(n, -127.0f), 127.0f);
    }
    __device__ static inline u32x2_t encode(const f32x8_t &x, float s)
    {
        const float inv = 1.0f / s;
        u32x2_t w;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            w[k] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[k] |= (uint32_t)(code(x[4 * k + e], s, inv) & 255) << (8 * e);
        }
        return w;
    }
    __device__ static inline f32x8_t decode(const u32x2_t &w)
    {
        f32x8_t x;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = (float)((int32_t)(w[e >> 2] << (24 - 8 * (e & 3))) >> 24);
        return x;
    }
};

struct CodeE4M3 {
    __device__ static inline float scale(uint32_t top)
    {
        // top = 1.f * 2^e: 2^(e-8) while 1.f <= 1.75, else 2^(e-7)
        const int32_t e = (int32_t)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u);
        return __builtin_bit_cast(float, (uint32_t)(e < 1 ? 1 : e) << 23);
    }
    __device__ static inline u32x2_t encode(const f32x8_t &x, float s)
    {
        const float inv = 1.0f / s;  // exact, and so are the products
        u32x2_t w;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            int32_t p = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * k] * inv, x[4 * k + 1] * inv, 0, false);
            w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * k + 2] * inv, x[4 * k + 3] * inv, p, true);
        }
        return w;
    }
    __device__ static inline f32x8_t decode(const u32x2_t &w)
    {
        f32x8_t x;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const f32x2_t a = __builtin_amdgcn_cvt_pk_f32_fp8((int32_t)w[k], false),
                          b = __builtin_amdgcn_cvt_pk_f32_fp8((int32_t)w[k], true);
            x[4 * k] = a[0], x[4 * k + 1] = a[1], x[4 * k + 2] = b[0], x[4 * k + 3] = b[1];
        }
        return x;
    }
};

}  // namespace im2win
