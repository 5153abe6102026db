// Argument checks shared by the host side of the block operators and of the layers: the current device, strides, and which
// address ranges meet.
#pragma once

#include <algorithm>
#include <initializer_list>

#include "../../include/linfusion_attn.h"
#include "host_util.h"

namespace lf {

// The current device and its SM count.
struct Here {
    int device, sms;
    linfusion_status_t st;
};
inline Here here()
{
    Here h = {0, 0, LINFUSION_OK};
    if (cudaGetDevice(&h.device) != cudaSuccess) {
        cudaGetLastError();
        h.st = LINFUSION_ERR_CUDA;
        return h;
    }
    h.sms = device_sm_count(h.device);
    if (h.sms == -2) h.st = LINFUSION_ERR_UNSUPPORTED;
    else if (h.sms < 0) h.st = LINFUSION_ERR_CUDA;
    return h;
}

inline linfusion_status_t end(cudaError_t e)
{
    if (e == cudaSuccess) return LINFUSION_OK;
    cudaGetLastError();
    return LINFUSION_ERR_CUDA;
}

// An axis of n rows, s elements apart: whole 16-byte pieces, and within 2^46 elements, so that sums of such reaches are exact.
// The stride of an axis of one row says nothing.
inline bool good_stride(int64_t n, int64_t s) { return n <= 1 || (s >= 0 && s % 8 == 0 && s <= (int64_t(1) << 46) / (n - 1)); }

// The bytes from the first to behind the last element that strides reach, as a half-open range.
struct Extent {
    const char* p;
    size_t bytes;
};
inline Extent extent(const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t row)
{
    const int64_t last = (n0 - 1) * s0 + (n1 - 1) * s1 + (n2 - 1) * s2 + row;
    return {static_cast<const char*>(p), static_cast<size_t>(last) * 2};
}
inline bool meet(const Extent& a, const Extent& b) { return overlaps(a.p, a.bytes, b.p, b.bytes); }

// Rows of `row` elements over axes of length n and stride s: no two of them share an element when, taken from the
// smallest stride to the largest, each stride steps over everything below it.  Axes of length one do not count.
struct Axis {
    int64_t n, s;
};
inline bool rows_disjoint(std::initializer_list<Axis> axes, int64_t row)
{
    Axis a[4];
    int count = 0;
    for (const Axis& x : axes)
        if (x.n > 1) a[count++] = x;
    std::sort(a, a + count, [](const Axis& x, const Axis& y) { return x.s < y.s; });
    int64_t reach = row;
    for (int i = 0; i < count; ++i) {
        if (a[i].s < reach) return false;
        reach += (a[i].n - 1) * a[i].s;
    }
    return true;
}

}  // namespace lf
