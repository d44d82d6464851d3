// Argument checks shared by the entry points: the thread's last error, ranges and
// their overlaps, and that each range is memory the current device can access.
#pragma once

#include "lh.h"

#include <hip/hip_runtime.h>

#include <stdarg.h>
#include <stdio.h>
#include <string.h>

namespace lh {
namespace check {

inline thread_local char g_last_error[512] = "";

inline lh_status fail(lh_status s, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return s;
}

struct Buf {
    const char* name;
    uintptr_t lo;
    uintptr_t hi;  // exclusive
};

inline bool overlaps(const Buf& a, const Buf& b)
{
    if (a.lo == a.hi || b.lo == b.hi) return false;  // empty ranges
    return a.lo < b.hi && b.lo < a.hi;
}

inline Buf buf(const char* name, const void* p, size_t bytes)
{
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    return Buf{name, lo, lo + bytes};
}

inline bool mul_ok(int64_t a, int64_t b, int64_t* out)
{
    return !__builtin_mul_overflow(a, b, out) && *out <= (INT64_C(1) << 60);
}

inline lh_status check_dtype(lh_dtype t)
{
    if (t != LH_F32 && t != LH_BF16)
        return fail(LH_ERR_UNSUPPORTED_DTYPE, "io_dtype %d is neither LH_F32 nor LH_BF16", (int)t);
    return LH_OK;
}

inline lh_status check_align(const Buf& b, uintptr_t a)
{
    if (b.lo % a != 0)
        return fail(LH_ERR_INVALID_ARG, "%s is not %u-byte aligned", b.name, (unsigned)a);
    return LH_OK;
}

inline lh_status check_device(int* dev)
{
    int n = 0;
    if (hipGetDeviceCount(&n) != hipSuccess || n < 1) {
        (void)hipGetLastError();
        return fail(LH_ERR_NO_DEVICE, "no HIP device is visible");
    }
    if (hipGetDevice(dev) != hipSuccess) {
        (void)hipGetLastError();
        return fail(LH_ERR_NO_DEVICE, "hipGetDevice failed");
    }
    return LH_OK;
}

// The range [lo, hi) must be memory the current device can access: device
// memory of this device, or pinned / managed host memory, and it must lie
// inside one allocation.  `seen` is the last allocation found accessible in the
// same call: a range inside it needs no further query (two runtime calls, about
// 0.3 us; a framework's small tensors share allocations).
inline lh_status check_accessible(const Buf& b, int dev, Buf* seen)
{
    if (b.lo == b.hi) return LH_OK;
    if (b.lo >= seen->lo && b.hi <= seen->hi) return LH_OK;
    void* p = reinterpret_cast<void*>(b.lo);
    hipPointerAttribute_t a;
    memset(&a, 0, sizeof(a));
    if (hipPointerGetAttributes(&a, p) != hipSuccess) {
        (void)hipGetLastError();
        return fail(LH_ERR_INVALID_ARG, "%s (%p) is not memory known to HIP", b.name, p);
    }
    if (a.type == hipMemoryTypeUnregistered)
        return fail(LH_ERR_INVALID_ARG, "%s (%p) is unregistered host memory", b.name, p);
    if (a.type == hipMemoryTypeDevice && a.device != dev)
        return fail(LH_ERR_INVALID_ARG, "%s lives on device %d, the current device is %d", b.name,
                    a.device, dev);
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipMemGetAddressRange(&base, &size, p) == hipSuccess && base != nullptr) {
        // compared as offsets from the base so that a reported size near
        // SIZE_MAX cannot wrap the allocation's end around
        const uintptr_t blo = reinterpret_cast<uintptr_t>(base);
        if (b.lo < blo || b.hi - blo > size)
            return fail(LH_ERR_INVALID_ARG,
                        "%s [%p, +%zu) extends past its allocation [%p, +%zu)", b.name, p,
                        (size_t)(b.hi - b.lo), base, size);
        if (size <= UINTPTR_MAX - blo) *seen = Buf{b.name, blo, blo + size};
    } else {
        (void)hipGetLastError();
    }
    return LH_OK;
}

// Every range of a call.
template <typename Range>
lh_status check_all_accessible(const Range& all, int dev)
{
    Buf seen{"", 0, 0};
    lh_status s;
    for (const Buf* b : all)
        if ((s = check_accessible(*b, dev, &seen)) != LH_OK) return s;
    return LH_OK;
}

inline lh_status from_hip(hipError_t e, const char* what)
{
    if (e == hipSuccess) return LH_OK;
    return fail(LH_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace check
}  // namespace lh
