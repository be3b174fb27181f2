// Internal definitions of the sequence operators (layer norm, relative
// position bias, attention): what their host side (seq_api.cpp) passes to the
// launches, and the element types' conversions.
#pragma once

#include "../../include/im2win_seq.h"
#include "common.hpp"

namespace im2win {

// Rows of the [rows][2][C] fp32 partial sums that the layer norm's backward
// call leaves for its reduction.
int64_t norm_partial_rows(int64_t rows, int64_t C);

hipError_t launch_norm_forward(const void *x, const void *w, const void *b, void *y, float *mean, float *rstd,
                               int64_t rows, int64_t C, int64_t x_stride, float eps, int dt, int wdt, hipStream_t st);
hipError_t launch_norm_backward(const void *dy, const void *x, const void *w, const float *mean, const float *rstd,
                                void *dx, void *dw, void *db, float *part, int64_t rows, int64_t C, int64_t dy_stride,
                                int64_t x_stride, int dt, int wdt, hipStream_t st);

// Buckets of the distances: the first m - e + 1 of `from` are the smallest n
// of buckets e .. m (from[m - e] = INT32_MAX, the last bucket has no end);
// below e the bucket is n itself.
constexpr int kMaxBuckets = 512;
struct Buckets {
    int32_t m, e, R, two;
    int32_t from[kMaxBuckets / 2 + 2];
};
Buckets make_buckets(int64_t buckets, int64_t R, int two_sided);

hipError_t launch_bias_forward(const Buckets &bk, const void *table, float *strip, int64_t H, int dt, hipStream_t st);
hipError_t launch_bias_backward(const Buckets &bk, const float *dstrip, void *dtable, int64_t n, int64_t H, int dt,
                                hipStream_t st);

// ---- element types: fp32 values in memory as fp32, fp16 or bf16 ----
struct EltF32 {
    typedef float T;
    __device__ static inline float get(T v) { return v; }
    __device__ static inline T put(float v) { return v; }
};
struct EltF16 {
    typedef _Float16 T;
    __device__ static inline float get(T v) { return (float)v; }
    __device__ static inline T put(float v) { return (T)v; }
};
struct EltBF16 {
    typedef __bf16 T;
    __device__ static inline float get(T v) { return (float)v; }
    __device__ static inline T put(float v) { return (T)v; }
};

}  // namespace im2win
