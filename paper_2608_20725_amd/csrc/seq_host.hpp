// Argument checks of the sequence operators on the host: buffers that lie in
// one device allocation, strided operands, and whether two of them meet.
#pragma once

#include "seq.hpp"

namespace im2win {
namespace {

constexpr int64_t kMaxLen = int64_t(1) << 20;
constexpr int64_t kMaxReach = int64_t(1) << 44;  // elements between the first and the last of an axis: no memory is larger

bool too_far(int64_t n, int64_t stride) { return n > 1 && stride > kMaxReach / (n - 1); }
bool known(int dt) { return dt == IM2WIN_F32 || dt == IM2WIN_F16 || dt == IM2WIN_BF16; }
int64_t elt(int dt) { return dt == IM2WIN_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t a) { return ((uintptr_t)p & (uintptr_t)(a - 1)) == 0; }
int64_t pad256(int64_t n) { return (n + 255) / 256 * 256; }

// A buffer of a call: the bytes from p on that it may touch.
struct Buf {
    const void *p;
    int64_t bytes;
};

// Checks that buffers lie in one device allocation each.  The allocations that
// a call has met are kept for its other buffers: asking the runtime takes 0.2
// us a buffer, and an allocator serves many tensors from one allocation.
class Extents {
public:
    int check(const Buf *b, int n)
    {
        for (int i = 0; i < n; ++i)
            if (b[i].bytes > 0)
                if (const int rc = one(b[i]))
                    return rc;
        return IM2WIN_OK;
    }

private:
    static constexpr int kMost = 8;
    uintptr_t base_[kMost];
    uint64_t size_[kMost];
    int n_ = 0;

    static bool inside(const Buf &b, uintptr_t base, uint64_t size)
    {
        const uintptr_t q = (uintptr_t)b.p;
        return q >= base && (uint64_t)(q - base) + (uint64_t)b.bytes <= size;
    }
    int one(const Buf &b)
    {
        for (int i = 0; i < n_; ++i)
            if (inside(b, base_[i], size_[i]))
                return IM2WIN_OK;
        hipDeviceptr_t base = nullptr;
        size_t size = 0;
        if (hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)b.p) != hipSuccess) {
            (void)hipGetLastError();  // leave no sticky error behind for the caller
            return IM2WIN_EBUFFER;
        }
        if (!inside(b, (uintptr_t)base, size))
            return IM2WIN_EBUFFER;
        if (n_ < kMost) {
            base_[n_] = (uintptr_t)base;
            size_[n_++] = size;
        }
        return IM2WIN_OK;
    }
};

bool meet(const Buf &a, const Buf &b) { return a.bytes > 0 && b.bytes > 0 && overlaps(a.p, a.bytes, b.p, b.bytes); }

// One operand [B][L][heads][D] in memory.
struct Operand {
    const void *p;
    int64_t B, L, heads, D, elt;
    int64_t stride[3];  // elements: sequence, token, head; 0 where there is one of them (or none): nothing steps

    Operand(const void *ptr, int64_t b, int64_t l, int64_t h, int64_t d, int64_t e, const int64_t *s)
        : p(ptr), B(b), L(l), heads(h), D(d), elt(e), stride{b > 1 ? s[0] : 0, l > 1 ? s[1] : 0, h > 1 ? s[2] : 0}
    {
    }
    int64_t bytes() const  // from the first element to the end of the last
    {
        if (B == 0 || L == 0)
            return 0;
        return ((B - 1) * stride[0] + (L - 1) * stride[1] + (heads - 1) * stride[2] + D) * elt;
    }
};

int check_strides(const Operand &o, bool any_token_stride = false)
{
    const int64_t n[3] = {o.B, o.L, o.heads};
    for (int k = 0; k < 3; ++k) {
        if (o.stride[k] < 0)
            return IM2WIN_EINVAL;
        if (too_far(n[k], o.stride[k]))
            return IM2WIN_ERANGE;
    }
    if (!any_token_stride && o.stride[1] * o.elt >= (int64_t)1 << 24)
        return IM2WIN_ERANGE;
    return IM2WIN_OK;
}

// Rows of an output must not meet each other: heads within a token, tokens
// within a sequence (or the other way round), sequences apart.
bool self_disjoint(const Operand &o)
{
    struct Axis {
        int64_t n, s;
    } ax[3] = {{o.B, o.stride[0]}, {o.L, o.stride[1]}, {o.heads, o.stride[2]}};
    for (int i = 0; i < 2; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (ax[j].s < ax[i].s) {
                const Axis t = ax[i];
                ax[i] = ax[j];
                ax[j] = t;
            }
    int64_t reach = o.D;  // elements one step of the next axis has to clear
    for (int i = 0; i < 3; ++i) {
        if (ax[i].n > 1 && ax[i].s < reach)
            return false;
        reach += (ax[i].n - 1) * ax[i].s;
    }
    return true;
}

// Bytes modulo `period` bytes that an operand takes from its first element on:
// the axes that step by whole periods add none.
int64_t width(const Operand &o, int64_t period)
{
    const int64_t n[3] = {o.B, o.L, o.heads};
    int64_t w = o.D;
    for (int k = 0; k < 3; ++k)
        if (n[k] > 1 && o.stride[k] * o.elt % period)
            w += (n[k] - 1) * o.stride[k];
    return w * o.elt;
}

// Two operands whose extents meet may still lie side by side, as q, k and v do
// in one tensor: there is a stride (the tokens', if they are columns of each
// token's row; the sequences' or heads' in other orders of the dimensions)
// modulo which their bytes are apart.
bool side_by_side(const Operand &a, const Operand &b)
{
    const int64_t n[6] = {a.B, a.L, a.heads, b.B, b.L, b.heads};
    const int64_t diff = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
    for (int k = 0; k < 6; ++k) {
        const int64_t period = k < 3 ? a.stride[k] * a.elt : b.stride[k - 3] * b.elt;
        if (n[k] <= 1 || period <= 0)
            continue;
        const int64_t off = ((diff % period) + period) % period;  // where b starts, a's start being 0
        if (off >= width(a, period) && off + width(b, period) <= period)
            return true;
    }
    return false;
}

bool clash(const Operand &a, const Operand &b)
{
    const Buf x{a.p, a.bytes()}, y{b.p, b.bytes()};
    return meet(x, y) && !side_by_side(a, b);
}

bool strides_aligned(const int64_t *s, int64_t B, int64_t L, int64_t heads, int64_t e)
{
    return (B <= 1 || s[0] * e % 16 == 0) && (L <= 1 || s[1] * e % 16 == 0) && (heads <= 1 || s[2] * e % 16 == 0);
}

}  // namespace
}  // namespace im2win
