// The learned relative position bias: bucket table -> strip by distance, and
// the strips' gradients back to the table's.
//
// A bucket is one contiguous range of distances on each side, so both
// directions are gathers (no atomics): the strip reads its bucket's entry,
// the table's gradient sums its bucket's range.  The bucket borders are found
// on the host in 64 bits and travel as a kernel argument.  Both are launch
// latency: a strip of 16 heads and 257 distances takes 3 us on the GPU, the
// gradient of 24 layers of 1601 distances and 320 buckets 5.
#include "seq.hpp"

#include <math.h>

namespace im2win {
namespace {

constexpr int kThreads = 256;

// strip[h][d + R] = table[bucket(d)][h]; a workgroup takes kThreads distances
// of one head.
template <class E>
__global__ __launch_bounds__(kThreads) void bias_fwd(Buckets bk, const typename E::T *__restrict__ table,
                                                     float *__restrict__ strip, int32_t H)
{
    const int i = blockIdx.x * kThreads + threadIdx.x, h = blockIdx.y;
    if (i > 2 * bk.R)
        return;
    const int d = i - bk.R;
    const int n = bk.two ? (d < 0 ? -d : d) : (d < 0 ? -d : 0);
    int b = n;
    if (n >= bk.e) {
        int lo = 0, hi = bk.m - bk.e;  // from[lo] <= n < from[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (bk.from[mid] <= n)
                lo = mid;
            else
                hi = mid;
        }
        b = bk.e + lo;
    }
    if (bk.two && d > 0)
        b += bk.m;
    strip[(int64_t)h * (2 * bk.R + 1) + i] = E::get(table[(int64_t)b * H + h]);
}

// One wave per bucket and head; its lanes take the (layer, distance) pairs of
// the bucket in a fixed order.
template <class E>
__global__ __launch_bounds__(kThreads) void bias_bwd(Buckets bk, const float *__restrict__ dstrip,
                                                     typename E::T *__restrict__ dtable, int32_t n, int32_t H)
{
    const int nb = bk.two ? 2 * bk.m : bk.m;
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y, lane = threadIdx.x & 63;
    if (b >= nb)
        return;
    const int k = b >= bk.m ? b - bk.m : b;  // bucket within its side
    // n = lo .. hi
    int lo = k, hi = k;
    if (k >= bk.e) {
        lo = bk.from[k - bk.e];
        hi = bk.from[k - bk.e + 1] - 1;
        if (hi > bk.R)
            hi = bk.R;
    }
    // distances first .. first + len - 1, as indices into the strip
    int first, len = hi - lo + 1;
    if (bk.two && b >= bk.m) {
        if (lo < 1)  // d = 0 belongs to the other side
            len -= 1 - lo, lo = 1;
        first = bk.R + lo;
    } else {
        first = bk.R - hi;
        if (!bk.two && lo == 0)  // the keys after the query too
            len += bk.R;
    }
    const int64_t W = 2 * bk.R + 1;
    float a = 0;
    if (len > 0)
        for (int l = lane; l < len * n; l += 64) {
            const int layer = l / len, o = l - layer * len;
            a += dstrip[((int64_t)layer * H + h) * W + first + o];
        }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1)
        a += __shfl_xor(a, m);
    if (lane == 0)
        dtable[(int64_t)b * H + h] = E::put(a);
}

}  // namespace

Buckets make_buckets(int64_t buckets, int64_t R, int two_sided)
{
    Buckets bk;
    bk.m = (int32_t)(two_sided ? buckets / 2 : buckets);
    bk.e = bk.m / 2;
    bk.R = (int32_t)R;
    bk.two = two_sided ? 1 : 0;
    const int far = bk.m - bk.e;
    const double step = log((double)R / bk.e) / far;
    bk.from[0] = bk.e;
    // floor(ln(n/e)/step + 1e-9) >= k from n = e*exp((k - 1e-9)*step) on
    for (int k = 1; k < far; ++k)
        bk.from[k] = (int32_t)ceil(bk.e * exp((k - 1e-9) * step));
    bk.from[far] = INT32_MAX;
    return bk;
}

hipError_t launch_bias_forward(const Buckets &bk, const void *table, float *strip, int64_t H, int dt, hipStream_t st)
{
    const dim3 g((uint32_t)((2 * bk.R + kThreads) / kThreads), (uint32_t)H);
    if (dt == IM2WIN_F32)
        bias_fwd<EltF32><<<g, kThreads, 0, st>>>(bk, (const float *)table, strip, (int32_t)H);
    else if (dt == IM2WIN_F16)
        bias_fwd<EltF16><<<g, kThreads, 0, st>>>(bk, (const _Float16 *)table, strip, (int32_t)H);
    else
        bias_fwd<EltBF16><<<g, kThreads, 0, st>>>(bk, (const __bf16 *)table, strip, (int32_t)H);
    return hipGetLastError();
}

hipError_t launch_bias_backward(const Buckets &bk, const float *dstrip, void *dtable, int64_t n, int64_t H, int dt,
                                hipStream_t st)
{
    const int nb = bk.two ? 2 * bk.m : bk.m;
    const dim3 g((uint32_t)((nb + 3) / 4), (uint32_t)H);
    if (dt == IM2WIN_F32)
        bias_bwd<EltF32><<<g, kThreads, 0, st>>>(bk, dstrip, (float *)dtable, (int32_t)n, (int32_t)H);
    else if (dt == IM2WIN_F16)
        bias_bwd<EltF16><<<g, kThreads, 0, st>>>(bk, dstrip, (_Float16 *)dtable, (int32_t)n, (int32_t)H);
    else
        bias_bwd<EltBF16><<<g, kThreads, 0, st>>>(bk, dstrip, (__bf16 *)dtable, (int32_t)n, (int32_t)H);
    return hipGetLastError();
}

}  // namespace im2win
