// Layer norm over the channels of each row, forward and backward.
//
// Both are one pass over the rows: a row is held in the registers of 8 to 1024
// lanes, so its two sums (mean, then the centred squares: no cancellation)
// cost no second read, and the backward pass keeps every lane's columns of
// dweight and dbias in registers over all the rows of its workgroup.  Rows
// that fit no register instance go through the looped kernels at the end.
// Memory-bound: 2 (3) elements moved a value.  Backward, 100352 rows of 512
// bf16 channels: 63 us, 4.9 TB/s, the rate of a large copy.
#include "seq.hpp"

namespace im2win {
namespace {

constexpr int kThreads = 256;

// Threads of a workgroup whose rows take LPR lanes each.
template <int LPR>
constexpr int threads() { return LPR < 256 ? 256 : LPR; }

// Sums of a and b over the row's LPR lanes (red: 2*LPR/64 floats where a row
// takes more than a wave, free again on return).
template <int LPR>
__device__ inline void row_sum2(float &a, float &b, float *red)
{
#pragma unroll
    for (int m = (LPR < 64 ? LPR : 64) / 2; m >= 1; m >>= 1) {
        a += __shfl_xor(a, m);
        b += __shfl_xor(b, m);
    }
    if constexpr (LPR > 64) {
        constexpr int N = LPR / 64;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            red[w] = a;
            red[N + w] = b;
        }
        __syncthreads();
        a = b = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            a += red[k];
            b += red[N + k];
        }
        __syncthreads();
    }
}

// n of VEC values from p as fp32 (n <= 0: none), the others `rest`.  Rows of odd
// length or stride start anywhere: the vectors are loaded and stored with
// their element's alignment, which is the same instruction for aligned
// addresses and hardly slower for others (5673 rows of 5112 fp16 channels
// forward: 38 us dense, 40 us 5115 apart, element by element 90 us).
template <class E, int VEC>
__device__ inline void load(const typename E::T *p, int n, float *f, float rest = 0.0f)
{
    typedef typename E::T V __attribute__((ext_vector_type(VEC), aligned(sizeof(typename E::T))));
    if (n >= VEC) {
        const V v = *(const V *)p;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            f[e] = E::get(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            f[e] = e < n ? E::get(p[e]) : rest;
    }
}

template <class E, int VEC>
__device__ inline void store(typename E::T *p, int n, const float *f)
{
    typedef typename E::T V __attribute__((ext_vector_type(VEC), aligned(sizeof(typename E::T))));
    if (n >= VEC) {
        V v;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            v[e] = E::put(f[e]);
        *(V *)p = v;
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (e < n)
                p[e] = E::put(f[e]);
    }
}

// A row of C <= LPR*NV*VEC values: vector i of a lane starts at column
// (i*LPR + lane)*VEC.
template <class E, class W, int VEC, int NV, int LPR>
__global__ __launch_bounds__((threads<LPR>())) void norm_fwd(const typename E::T *x,
                                                     const typename W::T *__restrict__ w,
                                                     const typename W::T *__restrict__ b, typename E::T *y,
                                                     float *__restrict__ mean, float *__restrict__ rstd, int64_t rows,
                                                     int32_t C, int64_t xs, float eps)
{
    __shared__ float red[LPR > 64 ? LPR / 32 : 1];
    constexpr int kRows = threads<LPR>() / LPR;
    const int lane = threadIdx.x % LPR;
    const float n = (float)C;
    float wv[NV][VEC], bv[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LPR + lane) * VEC;
        load<W, VEC>(w + c, C - c, wv[i]);
        load<W, VEC>(b + c, C - c, bv[i]);
    }
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR; r < rows;
         r += (int64_t)gridDim.x * kRows) {
        float v[NV][VEC];
        float s = 0, q = 0, unused = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LPR + lane) * VEC;
            load<E, VEC>(x + r * xs + c, C - c, v[i]);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                s += v[i][e];
        }
        row_sum2<LPR>(s, unused, red);
        const float mu = s / n;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int left = C - (i * LPR + lane) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v[i][e] -= mu;
                q += e < left ? v[i][e] * v[i][e] : 0.0f;
            }
        }
        row_sum2<LPR>(q, unused, red);
        const float rs = 1.0f / sqrtf(q / n + eps);
        if (lane == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LPR + lane) * VEC;
            float o[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                o[e] = v[i][e] * rs * wv[i][e] + bv[i][e];
            store<E, VEC>(y + r * C + c, C - c, o);
        }
    }
}

template <class E, class W, int VEC, int NV, int LPR>
__global__ __launch_bounds__((threads<LPR>())) void norm_bwd(const typename E::T *__restrict__ dy,
                                                     const typename E::T *__restrict__ x,
                                                     const typename W::T *__restrict__ w,
                                                     const float *__restrict__ mean, const float *__restrict__ rstd,
                                                     typename E::T *__restrict__ dx, float *__restrict__ part,
                                                     int64_t rows, int32_t C, int64_t dys, int64_t xs)
{
    __shared__ float red[LPR > 64 ? LPR / 32 : 1];
    extern __shared__ float cols[];  // more than one row at a time: [2][C]
    constexpr int kRows = threads<LPR>() / LPR;
    const int lane = threadIdx.x % LPR;
    const float inv = 1.0f / (float)C;
    float wv[NV][VEC], aw[NV][VEC], ab[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * LPR + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            aw[i][e] = ab[i][e] = 0;
        load<W, VEC>(w + c, C - c, wv[i]);
    }
    for (int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / LPR; r < rows;
         r += (int64_t)gridDim.x * kRows) {
        const float mu = mean[r], rs = rstd[r];
        float g[NV][VEC], h[NV][VEC];
        float s1 = 0, s2 = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LPR + lane) * VEC;
            // beyond the row dy is 0, and with it everything that is summed;
            // x is the mean there: 0 - mean times rstd may leave the range
            load<E, VEC>(dy + r * dys + c, C - c, g[i]);
            load<E, VEC>(x + r * xs + c, C - c, h[i], mu);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                h[i][e] = (h[i][e] - mu) * rs;
                aw[i][e] += g[i][e] * h[i][e];
                ab[i][e] += g[i][e];
                g[i][e] *= wv[i][e];
                s1 += g[i][e];
                s2 += g[i][e] * h[i][e];
            }
        }
        row_sum2<LPR>(s1, s2, red);
        s1 *= inv;
        s2 *= inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LPR + lane) * VEC;
            float o[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                o[e] = rs * (g[i][e] - s1 - h[i][e] * s2);
            store<E, VEC>(dx + r * C + c, C - c, o);
        }
    }
    // this workgroup's [2][C] sums: one row's lanes after the other add theirs
    float *out = part + (int64_t)blockIdx.x * 2 * C;
    if constexpr (kRows > 1) {
        for (int k = 0; k < kRows; ++k) {
            if ((int)(threadIdx.x / LPR) == k)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (i * LPR + lane) * VEC;
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (c + e < C) {
                            cols[c + e] = (k ? cols[c + e] : 0.0f) + aw[i][e];
                            cols[C + c + e] = (k ? cols[C + c + e] : 0.0f) + ab[i][e];
                        }
                }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * C; c += threads<LPR>())
            out[c] = cols[c];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * LPR + lane) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (c + e < C) {
                    out[c + e] = aw[i][e];
                    out[C + c + e] = ab[i][e];
                }
        }
    }
}

// Rows of any length, one workgroup a row: every pass reads the row again
// (from L2).  Rows that fit no register instance only.
template <class E, class W>
__global__ __launch_bounds__(kThreads) void norm_fwd_long(const typename E::T *x, const typename W::T *__restrict__ w,
                                                          const typename W::T *__restrict__ b, typename E::T *y,
                                                          float *__restrict__ mean, float *__restrict__ rstd,
                                                          int64_t rows, int32_t C, int64_t xs, float eps)
{
    __shared__ float red[8];
    const float n = (float)C;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        float s = 0, q = 0, unused = 0;
        for (int c = threadIdx.x; c < C; c += kThreads)
            s += E::get(x[r * xs + c]);
        row_sum2<256>(s, unused, red);
        const float mu = s / n;
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float d = E::get(x[r * xs + c]) - mu;
            q += d * d;
        }
        row_sum2<256>(q, unused, red);
        const float rs = 1.0f / sqrtf(q / n + eps);
        if (threadIdx.x == 0) {
            mean[r] = mu;
            rstd[r] = rs;
        }
        for (int c = threadIdx.x; c < C; c += kThreads)
            y[r * C + c] = E::put((E::get(x[r * xs + c]) - mu) * rs * W::get(w[c]) + W::get(b[c]));
    }
}

template <class E, class W>
__global__ __launch_bounds__(kThreads) void norm_bwd_long(const typename E::T *__restrict__ dy,
                                                          const typename E::T *__restrict__ x,
                                                          const typename W::T *__restrict__ w,
                                                          const float *__restrict__ mean,
                                                          const float *__restrict__ rstd, typename E::T *__restrict__ dx,
                                                          int64_t rows, int32_t C, int64_t dys, int64_t xs)
{
    __shared__ float red[8];
    const float inv = 1.0f / (float)C;
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float mu = mean[r], rs = rstd[r];
        float s1 = 0, s2 = 0;
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float g = E::get(dy[r * dys + c]) * W::get(w[c]);
            s1 += g;
            s2 += g * (E::get(x[r * xs + c]) - mu) * rs;
        }
        row_sum2<256>(s1, s2, red);
        for (int c = threadIdx.x; c < C; c += kThreads) {
            const float g = E::get(dy[r * dys + c]) * W::get(w[c]), h = (E::get(x[r * xs + c]) - mu) * rs;
            dx[r * C + c] = E::put(rs * (g - s1 * inv - h * s2 * inv));
        }
    }
}

// dweight and dbias of long rows: a lane sums one column over every
// gridDim.y-th row.
template <class E>
__global__ __launch_bounds__(kThreads) void norm_cols_long(const typename E::T *__restrict__ dy,
                                                           const typename E::T *__restrict__ x,
                                                           const float *__restrict__ mean,
                                                           const float *__restrict__ rstd, float *__restrict__ part,
                                                           int64_t rows, int32_t C, int64_t dys, int64_t xs)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= C)
        return;
    float aw = 0, ab = 0;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
        const float g = E::get(dy[r * dys + c]);
        aw += g * (E::get(x[r * xs + c]) - mean[r]) * rstd[r];
        ab += g;
    }
    float *out = part + (int64_t)blockIdx.y * 2 * C;
    out[c] = aw;
    out[C + c] = ab;
}

// Sums the partial rows: kCols columns a workgroup, each by 1024/kCols lanes
// that take the rows in turn, joined in a fixed order.  (16 columns rather
// than 32: twice the workgroups, 1024 columns of 1024 rows 11.3 -> 4.6 us.)
constexpr int kCols = 16;
template <class W>
__global__ __launch_bounds__(1024) void norm_reduce(const float *__restrict__ part, typename W::T *__restrict__ dw,
                                                    typename W::T *__restrict__ db, int32_t n, int32_t C)
{
    constexpr int N = 1024 / kCols;
    __shared__ float s[N][kCols + 1];
    const int cx = threadIdx.x % kCols, ry = threadIdx.x / kCols;
    const int64_t c = (int64_t)blockIdx.x * kCols + cx;
    float a = 0;
    if (c < 2 * (int64_t)C)
#pragma unroll 4
        for (int64_t r = ry; r < n; r += N)
            a += part[r * 2 * C + c];
    s[ry][cx] = a;
    __syncthreads();
    if (ry == 0 && c < 2 * (int64_t)C) {
        a = 0;
#pragma unroll
        for (int k = 0; k < N; ++k)
            a += s[k][cx];
        if (c < C)
            dw[c] = W::put(a);
        else
            db[c - C] = W::put(a);
    }
}

struct Args {
    const void *dy, *x, *w, *b;
    void *y;  // y or dx
    float *mean, *rstd;
    float *part;
    int64_t rows, C, dys, xs;
    float eps;
    hipStream_t st;
};

template <class E, class W, int VEC, int NV, int LPR>
void run(const Args &a, bool bwd)
{
    typedef typename E::T T;
    typedef typename W::T U;
    const int64_t rows_wg = threads<LPR>() / LPR;
    if (!bwd) {
        const int64_t want = (a.rows + rows_wg - 1) / rows_wg;
        const int64_t grid = want < 4096 ? want : 4096;
        norm_fwd<E, W, VEC, NV, LPR><<<(uint32_t)grid, threads<LPR>(), 0, a.st>>>(
            (const T *)a.x, (const U *)a.w, (const U *)a.b, (T *)a.y, a.mean, a.rstd, a.rows, (int32_t)a.C, a.xs,
            a.eps);
    } else {
        const size_t lds = rows_wg > 1 ? (size_t)a.C * 8 : 0;
        norm_bwd<E, W, VEC, NV, LPR><<<(uint32_t)norm_partial_rows(a.rows, a.C), threads<LPR>(), lds, a.st>>>(
            (const T *)a.dy, (const T *)a.x, (const U *)a.w, a.mean, a.rstd, (T *)a.y, a.part, a.rows, (int32_t)a.C,
            a.dys, a.xs);
    }
}

// The smallest instance that holds a row of C values; false when none does.
// Rows shorter than a wave's 64 vectors share the wave; long ones take up to
// 16 waves before a lane holds more than two vectors.  Between 257 and 1024
// vectors lanes of the forward pass hold more of them than those of the
// backward pass, which has three rows' worth of registers.  Measured, forward
// with 256, 512 and 1024 lanes: 5673 rows of 5112 fp16 channels 38.5, 41.6,
// 44.7 us, 20000x4096 bf16 62.7, 67.9, 60.6, 10000x8192 89, 84, 85, 5000x4096
// fp32 26.0, 25.5, 37.4; one wave for 4096 channels 137.  Backward: 5673x5112
// 94, 67, 57, 20000x4096 139, 159, 139, 10000x2048 fp32 53.3, 51.8, 53.2, 4
// rows of 4096 9.9, 9.4, 9.9, but 10000x8192 bf16 221, 238, 188.
template <class E, class W, int VEC>
bool run_held(const Args &a, bool bwd)
{
    const int64_t n = (a.C + VEC - 1) / VEC;  // vectors in a row
    if (n <= 8)
        run<E, W, VEC, 1, 8>(a, bwd);
    else if (n <= 16)
        run<E, W, VEC, 1, 16>(a, bwd);
    else if (n <= 32)
        run<E, W, VEC, 1, 32>(a, bwd);
    else if (n <= 64)
        run<E, W, VEC, 1, 64>(a, bwd);
    else if (n <= 128)
        run<E, W, VEC, 2, 64>(a, bwd);
    else if (n <= 256)
        run<E, W, VEC, 4, 64>(a, bwd);
    else if (n <= 512)
        bwd ? run<E, W, VEC, 1, 512>(a, bwd) : run<E, W, VEC, 2, 256>(a, bwd);
    else if (n <= 1024)
        bwd ? run<E, W, VEC, 2, 512>(a, bwd) : run<E, W, VEC, 4, 256>(a, bwd);
    else if (n <= 2048)
        run<E, W, VEC, 2, 1024>(a, bwd);
    else if (n <= 4096)
        run<E, W, VEC, 4, 1024>(a, bwd);
    else
        return false;
    return true;
}

template <class E, class W>
void run_typed(const Args &a, bool bwd, void *dw, void *db)
{
    typedef typename E::T T;
    typedef typename W::T U;
    const int32_t C = (int32_t)a.C;
    const int64_t grid = a.rows < 8192 ? a.rows : 8192;
    if (!run_held<E, W, 16 / sizeof(T)>(a, bwd)) {
        if (!bwd) {
            norm_fwd_long<E, W><<<(uint32_t)grid, kThreads, 0, a.st>>>((const T *)a.x, (const U *)a.w, (const U *)a.b,
                                                                       (T *)a.y, a.mean, a.rstd, a.rows, C, a.xs,
                                                                       a.eps);
        } else {
            if (grid)  // without rows the sums below are still to be written, as zeros
                norm_bwd_long<E, W><<<(uint32_t)grid, kThreads, 0, a.st>>>((const T *)a.dy, (const T *)a.x,
                                                                           (const U *)a.w, a.mean, a.rstd, (T *)a.y,
                                                                           a.rows, C, a.dys, a.xs);
            const dim3 g((uint32_t)((a.C + kThreads - 1) / kThreads), (uint32_t)norm_partial_rows(a.rows, a.C));
            norm_cols_long<E><<<g, kThreads, 0, a.st>>>((const T *)a.dy, (const T *)a.x, a.mean, a.rstd, a.part, a.rows,
                                                        C, a.dys, a.xs);
        }
    }
    if (bwd)
        norm_reduce<W><<<(uint32_t)((2 * a.C + kCols - 1) / kCols), 1024, 0, a.st>>>(
            a.part, (U *)dw, (U *)db, (int32_t)norm_partial_rows(a.rows, a.C), C);
}

hipError_t run_any(const Args &a, bool bwd, int dt, int wdt, void *dw, void *db)
{
    if (dt == IM2WIN_F32)
        run_typed<EltF32, EltF32>(a, bwd, dw, db);
    else if (dt == IM2WIN_F16)
        wdt == IM2WIN_F32 ? run_typed<EltF16, EltF32>(a, bwd, dw, db) : run_typed<EltF16, EltF16>(a, bwd, dw, db);
    else
        wdt == IM2WIN_F32 ? run_typed<EltBF16, EltF32>(a, bwd, dw, db) : run_typed<EltBF16, EltBF16>(a, bwd, dw, db);
    return hipGetLastError();
}

}  // namespace

int64_t norm_partial_rows(int64_t rows, int64_t C)
{
    // enough workgroups to fill 256 CUs; a workgroup takes one row at a time,
    // or four of the short ones, and with many rows at least 32.  Measured with
    // 256, 512, 1024 and 2048 workgroups: 100352x512 bf16 152, 94, 61, 74 us;
    // 500000x64 84, 57, 52, 74; 9765x771 fp32 28.6, 25.7, 26.2, 33.8 (the rule's
    // 306: 27.3); with 64, 128 and 256: 256x1024 bf16 12.0, 12.5, 13.2; 300x2000
    // fp16 22, 21, 23.  Long rows would take more: 20000x4096 bf16 159 (625),
    // 115 with 512 of them.
    const int64_t least = (rows + 31) / 32, step = C <= 1024 ? (rows + 3) / 4 : rows;
    const int64_t n = least > 256 ? least : step < 256 ? step : 256;
    return n < 1 ? 1 : n > 1024 ? 1024 : n;
}

hipError_t launch_norm_forward(const void *x, const void *w, const void *b, void *y, float *mean, float *rstd,
                               int64_t rows, int64_t C, int64_t x_stride, float eps, int dt, int wdt, hipStream_t st)
{
    const Args a{nullptr, x, w, b, y, mean, rstd, nullptr, rows, C, 0, x_stride, eps, st};
    return run_any(a, false, dt, wdt, nullptr, nullptr);
}

hipError_t launch_norm_backward(const void *dy, const void *x, const void *w, const float *mean, const float *rstd,
                                void *dx, void *dw, void *db, float *part, int64_t rows, int64_t C, int64_t dy_stride,
                                int64_t x_stride, int dt, int wdt, hipStream_t st)
{
    const Args a{dy,   x,    w, nullptr, dx,        const_cast<float *>(mean), const_cast<float *>(rstd),
                 part, rows, C, dy_stride, x_stride, 0.0f,                      st};
    return run_any(a, true, dt, wdt, dw, db);
}

}  // namespace im2win
