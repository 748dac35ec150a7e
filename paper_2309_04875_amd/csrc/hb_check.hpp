// Argument checks that the entry points share: what a buffer has to be, and the text of a HIP error.  No launches here.
#pragma once

#include "../../include/hb.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hb {

// Keeps the error's text for hb_last_hip_error and returns HB_EHIP.
int fail_hip(hipError_t e, const char *what);

struct Range {
    uintptr_t lo, hi;
};

inline Range range_of(const void *p, size_t n) { return Range{(uintptr_t)p, (uintptr_t)p + n * sizeof(int64_t)}; }

inline bool same(Range a, Range b) { return a.lo == b.lo; }
inline bool disjoint(Range a, Range b) { return a.hi <= b.lo || b.hi <= a.lo; }

// Allocations that the checks of ONE call have found to be this GPU's memory.  The buffers of a call mostly lie in a few
// allocations (a framework's allocator cuts many tensors out of one), and two queries of the HIP runtime for each of them
// were 0.2 us a buffer: 0.8 us of a call on one tensor, 12 us of one on 17.  Nothing is kept after the call.
struct KnownAllocations {
    static constexpr int kMost = 16;
    Range at[kMost];
    unsigned found = 0;                  // the newest kMost are kept
    int device = -1;                     // current device, once asked for
};

// The buffer must be memory the GPU can address, and [p, p + bytes) must lie inside one allocation.
inline int check_device_bytes(const void *p, size_t bytes, KnownAllocations &known)
{
    const Range r{(uintptr_t)p, (uintptr_t)p + bytes};
    for (unsigned i = 0; i < known.found && i < (unsigned)KnownAllocations::kMost; ++i) {
        const Range &a = known.at[i];
        if (r.lo >= a.lo && r.lo < a.hi) return r.hi <= a.hi ? HB_OK : HB_EINVAL;
    }
    hipPointerAttribute_t attr;
    hipError_t e = hipPointerGetAttributes(&attr, p);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return HB_EINVAL;  // not known to the HIP runtime: plain host memory or a wild pointer
    }
    switch (attr.type) {
    case hipMemoryTypeDevice:     // memory of another GPU is not addressable from the kernels launched here
        if ((known.device < 0 && hipGetDevice(&known.device) != hipSuccess) || attr.device != known.device) {
            (void)hipGetLastError();
            return HB_EINVAL;
        }
        break;
    case hipMemoryTypeManaged:
        break;
    case hipMemoryTypeHost:  // pinned host memory is usable only through its device-side address
        if (attr.devicePointer != p) return HB_EINVAL;
        break;
    default:  // unregistered host memory, arrays
        return HB_EINVAL;
    }
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    e = hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)p);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return HB_OK;  // allocation kinds without a queryable range: the attribute check has passed
    }
    const Range a{(uintptr_t)base, (uintptr_t)base + size};
    if (attr.type == hipMemoryTypeDevice) known.at[known.found++ % KnownAllocations::kMost] = a;
    return (r.lo >= a.lo && r.hi <= a.hi) ? HB_OK : HB_EINVAL;
}

inline int check_device_buffer(const void *p, size_t n, KnownAllocations &known) { return check_device_bytes(p, n * sizeof(int64_t), known); }

inline int check_common(const void *const *ptrs, int count, size_t n, KnownAllocations &known)
{
    if (n > HB_MAX_ELEMENTS) return HB_EINVAL;
    if (n == 0) return HB_OK;
    for (int i = 0; i < count; ++i) {
        if (ptrs[i] == nullptr) return HB_EINVAL;
    }
    for (int i = 0; i < count; ++i) {
        if (((uintptr_t)ptrs[i] & 7u) != 0) return HB_EALIGN;
    }
    for (int i = 0; i < count; ++i) {
        const int st = check_device_buffer(ptrs[i], n, known);
        if (st != HB_OK) return st;
    }
    return HB_OK;
}

// A device buffer of n floats with the given alignment.
inline int check_float_buffer(const void *p, size_t n, unsigned align, KnownAllocations &known)
{
    if (p == nullptr) return HB_EINVAL;
    if (((uintptr_t)p & (align - 1)) != 0) return HB_EALIGN;
    return check_device_bytes(p, n * sizeof(float), known);
}

// `count` device buffers of different sizes and alignments: those of no bytes are not looked at.
inline int check_buffers(const void *const *ptrs, const size_t *bytes, const unsigned *align, int count)
{
    for (int i = 0; i < count; ++i) {
        if (bytes[i] != 0 && ptrs[i] == nullptr) return HB_EINVAL;
    }
    for (int i = 0; i < count; ++i) {
        if (bytes[i] != 0 && ((uintptr_t)ptrs[i] & (align[i] - 1)) != 0) return HB_EALIGN;
    }
    KnownAllocations known;
    for (int i = 0; i < count; ++i) {
        const int st = bytes[i] != 0 ? check_device_bytes(ptrs[i], bytes[i], known) : HB_OK;
        if (st != HB_OK) return st;
    }
    return HB_OK;
}

// Whether each of the buffers first .. last - 1, those that a call writes, overlaps no other of the call.
inline bool outputs_disjoint(const void *const *ptrs, const size_t *bytes, int count, int first, int last)
{
    for (int o = first; o < last; ++o) {
        for (int i = 0; i < count; ++i) {
            if (i == o || bytes[i] == 0 || bytes[o] == 0) continue;
            const Range a{(uintptr_t)ptrs[o], (uintptr_t)ptrs[o] + bytes[o]}, b{(uintptr_t)ptrs[i], (uintptr_t)ptrs[i] + bytes[i]};
            if (!disjoint(a, b)) return false;
        }
    }
    return true;
}

}  // namespace hb
